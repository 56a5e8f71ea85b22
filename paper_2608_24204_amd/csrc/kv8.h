// The 8-bit key-value cache (storage type WICI_KV8) and the operators around it, as
// the host code and the kernels see them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"
#include "kernels.h"
#include "kv8_layout.h"

namespace wici {

constexpr float kKv8Least = 0x1p-60f;  // a row's largest magnitude counts as at least this

struct Kv8 {
  char* base;
  const int32_t* table;   // [n_seqs][max_pages], rows table_stride apart
  int64_t table_stride;
  int n_pages;            // of the pool: a table entry outside [0, n_pages) names no page
  int max_pages;          // table entries of a sequence
  int page_shift;
  int n_kv;
};

// The new rows of a launch: which sequence each belongs to and at which position.
enum Kv8RowsKind {
  KV8_ARRAYS,  // row_start (or one row a sequence) and length, device arrays
  KV8_CHUNK,   // one sequence: n_rows rows ending at position fixed_len - 1
  KV8_STATE,   // one row, at the position of `state`
  KV8_SEQS     // one row a sequence: pool, table and position from seqs
};
struct Kv8Rows {
  int kind;
  int n_seqs, n_rows;
  const int32_t* row_start;  // [n_seqs + 1] or nullptr
  const int32_t* length;     // [n_seqs]
  int fixed_len;
  const void* state;
  const SeqDesc* seqs;
  int layer;
};

// Head rows: element (row, head, d) at row * row_stride + head * head_stride + d.
struct HeadRows {
  void* p;  // nullptr: absent
  int bf16;
  int64_t row_stride, head_stride;
  // inputs of the append only: the rows are the sums, in order, of `n_sum` fp32 arrays
  // sum_stride elements apart (0 and 1: one array)
  int n_sum;
  int64_t sum_stride;
};

// Rotary tables: cos[pos][dim / 2].  layout 0 rotates (j, j + dim / 2), 1 (2j, 2j + 1);
// dimensions from dim on pass through.
struct RopeTab {
  const float* cos;  // nullptr: no rotation
  const float* sin;
  int n_pos, dim, layout;
};

// x[row, head] rotated at positions[row] into y (which may be x).
hipError_t launch_rope_rows(int hd, const HeadRows& x, const HeadRows& y, int n_rows, int n_heads,
                            const int32_t* positions, const RopeTab& rope, hipStream_t st);
// Fills cos / sin [n_pos][half] with factor * cos/sin(pos * freq[j]), angles in fp64.
struct RopeFreqs {
  double f[64];
  double factor;
};
hipError_t launch_rope_table(const RopeFreqs& f, int half, int64_t n_pos, float* cos, float* sin,
                             hipStream_t st);

// Appends rows: keys (rotated first when rope.cos is set) and values quantised into the
// cache; with q.p, the queries rotated and scaled by q_scale into q_out (which may be q).
hipError_t launch_kv8_append(int hd, const Kv8& c, const Kv8Rows& r, const RopeTab& rope, int n_q,
                             const HeadRows& q, const HeadRows& q_out, float q_scale,
                             const HeadRows& k, const HeadRows& v, hipStream_t st,
                             int edge = 3);
// The values of the rows' positions: k and v rows written (either may be absent).
hipError_t launch_kv8_read(int hd, const Kv8& c, const Kv8Rows& r, const HeadRows& k,
                           const HeadRows& v, hipStream_t st);

// Attention of the rows over the cache, causal: a row at position p sees positions <= p.
// Rows without positions (or whose pages are all absent) give zeros; rows of no sequence
// are left as they are.  `out` or (out.p == nullptr) `act`, row t at t * n_q * hd.
struct Kv8Attn {
  int hd, n_q;
  float scale;
  HeadRows q, out;
  ActBuf act;
  int max_rows, max_length;  // the most rows / positions expected of a sequence
  float* work;               // kv8_attn_floats floats
};
size_t kv8_attn_floats(int hd, int n_q, int n_kv, int n_seqs, int n_rows, int max_rows,
                       int max_length);
size_t kv8_attn_floats_most(int hd);  // of any launch
// (edge: which of the timer's events the launches of append and attention record)
hipError_t launch_kv8_attn(const Kv8& c, const Kv8Rows& r, const Kv8Attn& a, hipStream_t st,
                           int edge = 3);

#ifdef __HIPCC__
// One sequence of a launch.
struct Kv8Seq {
  char* base;
  const int32_t* table;
  int row0, rows;  // its new rows
  int len;         // positions, the new rows included
};
__device__ __forceinline__ Kv8Seq kv8_seq(const Kv8& c, const Kv8Rows& r, int b) {
  Kv8Seq s;
  s.base = c.base;
  s.table = c.table + (int64_t)b * c.table_stride;
  s.row0 = b;
  s.rows = 1;
  if (r.kind == KV8_ARRAYS) {
    if (r.row_start) {
      kv8_range(r.row_start[b], r.row_start[b + 1], r.n_rows, s.row0, s.rows);
    }
    s.len = max(r.length[b], 0);
  } else if (r.kind == KV8_CHUNK) {
    s.row0 = 0;
    s.rows = r.n_rows;
    s.len = r.fixed_len;
  } else if (r.kind == KV8_STATE) {
    s.len = static_cast<const DecodeState*>(r.state)->pos + 1;
  } else {
    const SeqDesc sd = r.seqs[b];
    s.base = static_cast<char*>(sd.kv) + (size_t)r.layer * sd.kv_layer_stride;
    s.table = sd.table;
    s.len = static_cast<const DecodeState*>(sd.state)->pos + 1;
  }
  return s;
}
#endif

}  // namespace wici
