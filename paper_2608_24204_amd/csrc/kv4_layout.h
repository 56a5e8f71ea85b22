// Layout of the 4-bit key-value cache.  Plain arithmetic, so that a test can evaluate it on the
// CPU; pages, rows and positions are bounded as for the 8-bit cache.
#pragma once
#include "kv8_layout.h"

namespace wici {

constexpr int kKv4Group = 32;       // dimensions that share a scale
constexpr int kKv4LeastByte = 67;   // scales are 2^(byte - 127): 2^-60 ..
constexpr int kKv4MostByte = 252;   // .. 2^125
constexpr int kKv4NanByte = 255;    // of a row that is not finite

// A block (one page, keys or values, one KV head) is page * hd / 2 bytes of codes, then page *
// hd / 32 scale bytes.  A byte of codes holds dimensions 2 j (low bits) and 2 j + 1.  Key bytes lie
// position by position, and so do their scales: a lane of the attention takes 32 (heads of 64: 16)
// dimensions of one position.  Value bytes lie in groups of four positions, the four of a pair of
// dimensions side by side, and so do their scales: a lane takes four positions of 8 (4) dimensions.
// No byte belongs to two positions, so rows are appended by byte stores alone.
WICI_HD size_t kv4_block_bytes(int page, int hd) { return (size_t)page * (hd / 2 + hd / kKv4Group); }
WICI_HD size_t kv4_block_at(int phys, int which, int h, int n_kv, int page, int hd) {
  return (((size_t)phys * 2 + which) * n_kv + h) * kv4_block_bytes(page, hd);
}
// (the byte of dimension d)
WICI_HD int kv4_key_at(int slot, int d, int hd) { return slot * (hd / 2) + (d >> 1); }
WICI_HD int kv4_value_at(int slot, int d, int hd) {
  return (slot >> 2) * 2 * hd + 4 * (d >> 1) + (slot & 3);
}
WICI_HD int kv4_key_scale_at(int slot, int group, int page, int hd) {
  return page * (hd / 2) + slot * (hd / kKv4Group) + group;
}
WICI_HD int kv4_value_scale_at(int slot, int group, int page, int hd) {
  return page * (hd / 2) + (slot >> 2) * 4 * (hd / kKv4Group) + 4 * group + (slot & 3);
}

// The scale byte of dimensions whose largest magnitude has these bits (finite): the least exponent
// e with that at most 7 2^e.  The largest codes are 4 and 6, a step of 2 apart, so that up to 7 no
// value is further from its code than half that step.
WICI_HD int kv4_scale_byte(uint32_t most) {
  // most = m 2^x with m in [1, 2): e = x - 2 up to m = 1.75 (mantissa 0x600000), else x - 1
  const int byte = (int)((most + 0x1fffffu) >> 23) - 2;
  return byte < kKv4LeastByte ? kKv4LeastByte : byte > kKv4MostByte ? kKv4MostByte : byte;
}

}  // namespace wici
