// Layout of the paged cache's keys and values.
//
// A page holds P = page_size tokens (a power of two, at least 32) of every kv head:
// [pages][heads] records of P * dim elements, in the order in which the attention's MFMA
// operands take them, so that a wavefront loads a fragment as 1 KB side by side, straight
// into registers.  Everything is made of pieces of 16 bytes:
//   keys    tiles of 16 tokens: [tile][piece of the row][token], a piece 8 (16-bit rows) or
//           16 (codes) consecutive elements of a row
//   values  blocks of 32 tokens, transposed: 16-bit [block][16 elements][q][element][8 tokens],
//           codes [block][32 elements][q][element % 16][element / 16][8 tokens].  The 8 tokens
//           of q are 4 q .. 4 q + 3 and 16 + 4 q .. 16 + 4 q + 3: the scores of two key tiles
//           leave the MFMA with just those tokens in lane quarter q, so the weights enter
//           the second product without moving between lanes.
// Scales (8-bit codes): fp32 [pages][heads][P] for keys and for values.
#pragma once
#include "mxmoe_internal.h"

namespace mxmoe {

// Byte offset, inside a page's record of one head, of elements 8 c .. 8 c + 7 of the key
// of token t (side by side), and of element d of the value of token t.
template <int ES> __device__ __forceinline__ int key_at(int t, int c, int dim) {
  if (ES == 2) return ((t >> 4) * (dim / 8) + c) * 256 + (t & 15) * 16;
  return ((t >> 4) * (dim / 16) + (c >> 1)) * 256 + (t & 15) * 16 + (c & 1) * 8;
}
template <int ES> __device__ __forceinline__ int value_at(int t, int d, int dim) {
  const int q = (t >> 2) & 3, j = (t & 3) + ((t >> 4) & 1) * 4;
  if (ES == 2) return (((t >> 5) * (dim / 16) + (d >> 4)) * 4 + q) * 256 + (d & 15) * 16 + 2 * j;
  return (((t >> 5) * (dim / 32) + (d >> 5)) * 4 + q) * 256 + (d & 15) * 16 + ((d >> 4) & 1) * 8 + j;
}

}  // namespace mxmoe
