// Head rows as the kernels that append to a paged cache and read it back take them: a row of hd
// values is a unit of hd / 8 lanes, eight values a lane; its rotation, its place in the cache.
#pragma once
#include "kv8.h"
#include "launch.h"

namespace wici {

// Four consecutive elements at element offset `at` (a multiple of 4).
__device__ __forceinline__ void load4(const HeadRows& x, int64_t at, float* o) {
  if (x.bf16) {
    const uint2 v = *reinterpret_cast<const uint2*>(static_cast<const bf16_t*>(x.p) + at);
    o[0] = __uint_as_float(v.x << 16); o[1] = __uint_as_float(v.x & 0xffff0000u);
    o[2] = __uint_as_float(v.y << 16); o[3] = __uint_as_float(v.y & 0xffff0000u);
  } else {
    const float4 v = *reinterpret_cast<const float4*>(static_cast<const float*>(x.p) + at);
    o[0] = v.x; o[1] = v.y; o[2] = v.z; o[3] = v.w;
  }
}
__device__ __forceinline__ void put4(const HeadRows& x, int64_t at, const float* v) {
  if (x.bf16) {
    *reinterpret_cast<uint2*>(static_cast<bf16_t*>(x.p) + at) =
        make_uint2((uint32_t)f32_to_bf16(v[0]) | ((uint32_t)f32_to_bf16(v[1]) << 16),
                   (uint32_t)f32_to_bf16(v[2]) | ((uint32_t)f32_to_bf16(v[3]) << 16));
  } else {
    *reinterpret_cast<float4*>(static_cast<float*>(x.p) + at) = make_float4(v[0], v[1], v[2], v[3]);
  }
}

// Eight: runs a and b of four, as one where they are consecutive.
__device__ __forceinline__ void load44(const HeadRows& x, int64_t at, int a, int b, float (&o)[8]) {
  if (x.bf16 && b == a + 4) {
    load8(static_cast<const bf16_t*>(x.p) + at + a, o);
  } else {
    load4(x, at + a, o);
    load4(x, at + b, o + 4);
  }
}
__device__ __forceinline__ void put44(const HeadRows& x, int64_t at, int a, int b,
                                      const float (&v)[8]) {
  if (x.bf16 && b == a + 4) {
    uint4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      (&w.x)[i] = (uint32_t)f32_to_bf16(v[2 * i]) | ((uint32_t)f32_to_bf16(v[2 * i + 1]) << 16);
    *reinterpret_cast<uint4*>(static_cast<bf16_t*>(x.p) + at + a) = w;
  } else {
    put4(x, at + a, v);
    put4(x, at + b, v + 4);
  }
}

// The eight dimensions of lane c of a unit, as two runs of four: consecutive, or (a
// rotated run of the half layout) the first members of four pairs and the second.
struct Runs {
  int a, b;
  bool turn;  // rotated
};
__device__ __forceinline__ Runs runs(const RopeTab& rope, int c) {
  Runs r{8 * c, 8 * c + 4, false};
  if (rope.cos && 8 * c < rope.dim) {
    r.turn = true;
    if (rope.layout == 0) {
      r.a = 4 * c;
      r.b = rope.dim / 2 + 4 * c;
    }
  }
  return r;
}

// (a, b) -> (a cos - b sin, a sin + b cos) for each pair, every product and sum rounded
// to fp32 by itself: the codes of a rotated key are then a function of the row alone
// and not of how a compiler joins the products.
__device__ __forceinline__ void turn8(float (&x)[8], const float4& c, const float4& s, int layout) {
#pragma clang fp contract(off)
  const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float& u = layout ? x[2 * i] : x[i];
    float& w = layout ? x[2 * i + 1] : x[4 + i];
    const float a = u, b = w;
    const float ac = a * cc[i], bs = b * ss[i], as = a * ss[i], bc = b * cc[i];
    u = ac - bs;
    w = as + bc;
  }
}

// A unit's rotation at position pos; past the table the row is NaN (no angle is known).
__device__ __forceinline__ void turn_row(const RopeTab& rope, const Runs& r, int c, int pos,
                                         float (&x)[8]) {
  if (!r.turn) return;
  const size_t at = (size_t)min(pos, rope.n_pos - 1) * (rope.dim / 2) + 4 * c;
  const float4 cs = *reinterpret_cast<const float4*>(rope.cos + at);
  const float4 sn = *reinterpret_cast<const float4*>(rope.sin + at);
  turn8(x, cs, sn, rope.layout);
  if (pos >= rope.n_pos) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(0x7fc00000u);
  }
}

// The largest of a unit's values as bits: for magnitudes the order of the bits is the
// order of the values, and infinities and NaN come out above every finite one.
template <int LPU>
__device__ __forceinline__ unsigned unit_max(unsigned v) {
#pragma unroll
  for (int m = LPU / 2; m >= 1; m >>= 1) v = max(v, (unsigned)__shfl_xor((int)v, m));
  return v;
}

// Sequence and position of row t: found by counting the sequences that start at or
// before it, the unit's lanes side by side.
struct RowAt {
  bool there;
  char* base;
  const int32_t* table;
  int pos;
  int end;  // the row after the sequence's last
};
template <int LPU>
__device__ __forceinline__ RowAt row_at(const Kv8& c, const Kv8Rows& r, int t, int lane) {
  int b = t;
  if (r.kind == KV8_ARRAYS && r.row_start) {
    int n = 0;
    for (int j = lane; j <= r.n_seqs; j += LPU) n += r.row_start[j] <= t;
#pragma unroll
    for (int m = LPU / 2; m >= 1; m >>= 1) n += __shfl_xor(n, m);
    b = n - 1;
  } else if (r.kind == KV8_CHUNK) {
    b = 0;
  }
  if (b < 0 || b >= r.n_seqs) return RowAt{false, nullptr, nullptr, 0, 0};
  const Kv8Seq s = kv8_seq(c, r, b);
  const int pos = s.len - s.rows + (t - s.row0);
  return RowAt{t < s.row0 + s.rows && pos >= 0, s.base, s.table, pos, s.row0 + s.rows};
}
// The places of R neighbouring rows from t on: found once for those of one sequence.
template <int LPU, int R>
__device__ __forceinline__ void rows_at(RowAt (&w)[R], const Kv8& c, const Kv8Rows& r, int t,
                                        int lane) {
  w[0] = row_at<LPU>(c, r, t, lane);
#pragma unroll
  for (int i = 1; i < R; ++i) {
    if (w[i - 1].there && t + i < w[i - 1].end) {
      w[i] = w[i - 1];
      w[i].pos += 1;
    } else {
      w[i] = t + i < r.n_rows ? row_at<LPU>(c, r, t + i, lane)
                              : RowAt{false, nullptr, nullptr, 0, 0};
    }
  }
}
// Whether R rows are the R positions of one word of value codes (in a page that exists).
template <int R>
__device__ __forceinline__ bool one_word(const RowAt (&w)[R], char* const (&blk)[R]) {
  return R == 4 && blk[0] && (w[0].pos & 3) == 0 && w[R - 1].there && w[R - 1].end == w[0].end &&
         w[R - 1].table == w[0].table && w[R - 1].pos == w[0].pos + R - 1;
}

// ------------------------------------------------------------------- launch sizes
// Workgroups of `units` units, or 0 when there are none or 2^28 and more (16 threads each, of
// 2^32 in a grid).
inline unsigned unit_blocks(int hd, int64_t units) {
  const int64_t per = 256 / (hd / 8), n = (units + per - 1) / per;
  return units < 1 || units >= (int64_t)1 << 28 ? 0 : (unsigned)n;
}

// Rows a unit takes: four of a prompt, one where rows are few or belong to as many sequences.
inline int rows_of_unit(const Kv8Rows& r) { return r.n_rows >= 64 && r.n_rows >= 4 * r.n_seqs ? 4 : 1; }

}  // namespace wici
