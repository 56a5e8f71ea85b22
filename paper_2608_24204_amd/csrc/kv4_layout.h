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

// A row's reference is set so that its largest weight is 2^top, and moves before a lane's eight weights
// sum up to more than most = 2^log_most.
struct Room {
  float top, most;
  int log_most;
};
// fp16 weights: 2^14 fits, and fp16's least step is 2^-30 of the largest weight.
constexpr Room kRoomHalf{6.f, 0x1p14f, 14}, kRoomBf16{0.f, 0x1p8f, 8};

// Once a wavefront has met large values its rows' outputs hold 2^-lift of their sums, for which the
// weights are multiplied by that.  (Not by other references: those of large scores are too coarse to
// hold such a shift.)  n <= 2^lg positions add up to at most 2^(lg - 3) most times the largest value, 6
// times the largest scale.
//  - Values are large from a scale of 2^e on that leaves 2^(lg - 3) most 6 2^(e - 1) below 2^127: e = 128 -
//    log_most - lg; at most 2^100, which contexts of 2^14 positions need (2^20 for weights in bf16).  The
//    joins take what is not lifted by factors of at most 1.
//  - With the largest scale, 2^125, 2^(lg - 3 - lift) most 6 2^125 is below 2^126 for lift = lg + log_most -
//    1; contexts below 2^25 positions take that of 2^25.  Two joins, of wavefronts and of splits, take
//    what is lifted by less than 2 each, where the largest reference is that of an output that is not.
WICI_HD int kv4_log_of(int n) { return n < 2 ? 1 : 32 - __builtin_clz((unsigned)n - 1u); }
WICI_HD int kv4_large_byte(const Room& room, int n) {
  const int e = 128 - room.log_most - kv4_log_of(n);
  return 127 + (e < 100 ? e : 100);
}
WICI_HD int kv4_lift(const Room& room, int n) {
  const int lg = kv4_log_of(n);
  return (lg < 25 ? 25 : lg) + room.log_most - 1;
}

}  // namespace wici
