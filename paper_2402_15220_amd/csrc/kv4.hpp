// The 4-bit K/V tile of a KV4 cache, shared by the host and the kernels.
//
// A row of D elements of one token and head stands for low + scale * code:
// low = the row's minimum, scale = fp16((max - low) / 15), codes 0..15, both
// parameters fp16. One (slot, head) tile of K, or of V, is kv4_tile_bytes():
// kv4_rows(C) rows of codes, D/2 bytes each, then one (scale, low) pair of
// fp16 a row. Codes come in blocks of 16 tokens, laid out as the kernels'
// matrix operands need them:
//   K  token-major: the 32-bit word W of a row holds elements 8W .. 8W + 7.
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

}  // namespace ca
