// The 4-bit K/V tile of a KV4 cache, shared by the host and the kernels.
//
// A row of D elements of one token and head stands for low + scale * code:
// low = the row's minimum, scale = fp16((max - low) / 15), codes 0..15, both
// parameters fp16. One (slot, head) tile of K, or of V, is kv4_tile_bytes():
// kv4_rows(C) rows of codes, D/2 bytes each, then one (scale, low) pair of
// fp16 a row. Codes come in blocks of 16 tokens, laid out as the kernels'
// matrix operands need them:
//   K  word (16 g + n) * D/32 + w holds elements 8W .. 8W + 7 of token n,
//      W = g * D/32 + w: lane 16 g + n of a wavefront reads its D/32 words at
//      once, and a wavefront's load is one run of memory.
//   V  for group g = token % 16 / 4, channel n of each 16 and pair t of
//      16-channel tiles, word (16 g + n) * D/32 + t holds the codes of the
//      group's four tokens at channels 32 t + n and 32 t + 16 + n.
// Inside a word, element k (K: element 8W + k; V: token i of the group at
// channel 32 t + 16 b + n is k = 4 b + i) sits at nibble (k >> 1) + 4 (k & 1),
// so (word >> 8b) & 0x000f000f and & 0x00f000f0 are two pairs of neighbours
// in the halves of a register each.
#pragma once

#include <cstddef>
#include <cstdint>

namespace ca {

constexpr int kv4_rows(int C) { return (C + 15) / 16 * 16; }
constexpr int64_t kv4_tile_bytes(int C, int D) {
  return static_cast<int64_t>(kv4_rows(C)) * (D / 2 + 4);
}
constexpr int kv4_nibble(int k) { return (k >> 1) + 4 * (k & 1); }
// word of elements 8W .. 8W + 7 of K token t, counted from the tile's start
constexpr int kv4_k_word(int t, int W, int D) {
  return (t & ~15) * (D / 8) + (16 * (W / (D / 32)) + (t & 15)) * (D / 32) + W % (D / 32);
}

}  // namespace ca
