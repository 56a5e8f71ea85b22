// Layout of the 8-bit key-value cache and the bounds that its kernels put on what device
// memory tells them (page tables, lengths, row ranges).  Plain arithmetic, so that a test
// can evaluate it on the CPU.
#pragma once
#include <cstddef>
#include <cstdint>

#if defined(__HIPCC__)
#define WICI_HD __host__ __device__ __forceinline__
#else
#define WICI_HD inline
#endif

namespace wici {

// A block (one page, keys or values, one KV head) is page * hd codes, then page fp32
// scales, one for each position; a value is (code - 128) * scale.  Key codes lie position
// by position; value codes in groups of four positions, the four codes of a dimension
// side by side: a lane of the attention that multiplies four positions of one dimension
// reads them as one word.  Blocks follow each other as [page][keys, values][KV head].
WICI_HD size_t kv8_block_bytes(int page, int hd) { return (size_t)page * (hd + 4); }
WICI_HD size_t kv8_block_at(int phys, int which, int h, int n_kv, int page, int hd) {
  return (((size_t)phys * 2 + which) * n_kv + h) * kv8_block_bytes(page, hd);
}
WICI_HD int kv8_key_at(int slot, int d, int hd) { return slot * hd + d; }
WICI_HD int kv8_value_at(int slot, int d, int hd) {
  return (slot >> 2) * 4 * hd + 4 * d + (slot & 3);
}
WICI_HD int kv8_scale_at(int slot, int page, int hd) { return page * hd + 4 * slot; }

// The page holding logical page p of a sequence, or -1: past the sequence's table, or an
// entry that names no page of the pool.
WICI_HD int kv8_page(const int32_t* table, int64_t p, int max_pages, int n_pages) {
  if (p < 0 || p >= max_pages) return -1;
  const int phys = table[p];
  return phys < 0 || phys >= n_pages ? -1 : phys;
}

// The same in two parts, for a look-up whose answer is wanted later: the entry to read (p below
// 2^32, max_pages at least 1; past the table the last one, whose page then stands for positions
// that no row sees), and the page it names or -1.
WICI_HD uint32_t kv8_entry(uint32_t p, int max_pages) {
  return p < (uint32_t)max_pages ? p : (uint32_t)max_pages - 1;
}
WICI_HD int kv8_named(int entry, int n_pages) {
  return (uint32_t)entry < (uint32_t)n_pages ? entry : -1;
}

// The rows a sequence has when row_start says [from, to): a range inside [0, n_rows].
WICI_HD void kv8_range(int from, int to, int n_rows, int& row0, int& rows) {
  row0 = from < 0 ? 0 : from > n_rows ? n_rows : from;
  rows = (to < row0 ? row0 : to > n_rows ? n_rows : to) - row0;
}

// Positions that row i of `rows` new rows sees: those up to its own (len - rows + i), of
// a cache of `cap` positions; none for a row at a negative position.
WICI_HD int kv8_seen(int len, int rows, int i, int64_t cap) {
  const int64_t n = (int64_t)len - rows + i + 1;
  return (int)(n < 0 ? 0 : n > cap ? cap : n);
}

// Steps of `step` positions that hold n (0 .. 2^31 - 1).
WICI_HD int kv8_steps(int n, int step) {
  return (int)(((uint32_t)n + (uint32_t)step - 1) / (uint32_t)step);
}

// Floats of the partial results of a launch that splits its positions (parts: rows x heads x
// splits): their outputs, hd floats each, and behind all outputs their states (ref, lift, sum and
// one float that is not used): each is as aligned as the workspace, for any number of parts.
WICI_HD size_t kv8_part_out(size_t part, int hd) { return part * hd; }
WICI_HD size_t kv8_part_state(size_t part, size_t parts, int hd) { return parts * hd + 4 * part; }
WICI_HD size_t kv8_part_floats(size_t parts, int hd) { return parts * (hd + 4); }

}  // namespace wici
