// Rotary positions, and the 8-bit key-value cache as it is written and read back.
//
// Each row is read once and written once.  A head row of hd values is a unit of hd / 8
// lanes, eight values a lane, so a unit's maximum is a reduction within its lanes and no unit
// waits for another.
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

// ------------------------------------------------------------------- rotary positions
// The table is read where another head of the row has read it before; a row's heads are
// neighbouring units.  Bound by memory: 8192 rows of 32 heads of 128 (bf16, pairs) 24 us for 134
// MB, 5.6 TB/s where a large copy moves 5.2 (8 bytes a lane at a time: 26), on inputs partly in
// the memory-side cache; in calls whose inputs change 28.7 us, 4.7 TB/s.  32 rows 3.2 us.
template <int HD>
__global__ __launch_bounds__(256) void k_rope_rows(HeadRows x, HeadRows y, int n_rows, int n_heads,
                                                   const int32_t* __restrict__ positions,
                                                   RopeTab rope) {
  constexpr int LPU = HD / 8, UPB = 256 / LPU;
  const unsigned u = blockIdx.x * UPB + threadIdx.x / LPU;  // below 2^28
  const int c = threadIdx.x % LPU;
  const int row = (int)(u / n_heads), h = (int)(u % n_heads);
  if (row >= n_rows) return;
  const int pos = positions[row];
  if (pos < 0) return;  // padding: left as it is
  const Runs r = runs(rope, c);
  float v[8];
  const int64_t in = row * x.row_stride + h * x.head_stride;
  load44(x, in, r.a, r.b, v);
  turn_row(rope, r, c, pos, v);
  put44(y, row * y.row_stride + h * y.head_stride, r.a, r.b, v);
}

// bf16 rows of the half layout, 16 dimensions of it at a time turned: two runs of eight a
// lane, so that they too are read and written 16 bytes a lane (calls of the same 8192 rows, all turned,
// take 28 us, with runs of four 34).
template <int HD>
__global__ __launch_bounds__(256) void k_rope_halves(HeadRows x, HeadRows y, int n_rows, int n_heads,
                                                     const int32_t* __restrict__ positions,
                                                     RopeTab rope) {
  constexpr int LPU = HD / 16, UPB = 256 / LPU;
  const unsigned u = blockIdx.x * UPB + threadIdx.x / LPU;  // below 2^28
  const int c = threadIdx.x % LPU;
  const int row = (int)(u / n_heads), h = (int)(u % n_heads);
  if (row >= n_rows) return;
  const int pos = positions[row];
  if (pos < 0) return;  // padding: left as it is
  const bool turn = 16 * c < rope.dim;
  const int a = turn ? 8 * c : 16 * c, b = turn ? rope.dim / 2 + 8 * c : 16 * c + 8;
  const bf16_t* from = static_cast<const bf16_t*>(x.p) + row * x.row_stride + h * x.head_stride;
  float v[16];
  load8(from + a, v);
  load8(from + b, v + 8);
  if (turn) {
    // four pairs at a time, as turn_row takes them
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float p[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        p[j] = v[4 * i + j];
        p[4 + j] = v[8 + 4 * i + j];
      }
      turn_row(rope, Runs{0, 0, true}, 2 * c + i, pos, p);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[4 * i + j] = p[j];
        v[8 + 4 * i + j] = p[4 + j];
      }
    }
  }
  const int64_t out = row * y.row_stride + h * y.head_stride;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float p[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = v[8 * i + j];
    put44(y, out, i ? b : a, (i ? b : a) + 4, p);
  }
}

__global__ __launch_bounds__(256) void k_rope_table(RopeFreqs f, int half, int64_t n,
                                                    float* __restrict__ cos_t,
                                                    float* __restrict__ sin_t) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  // angles of far positions need more than fp32: at position 100000 its step is 2^-7
  const double a = (double)(i / half) * f.f[i % half];
  cos_t[i] = (float)(f.factor * cos(a));
  sin_t[i] = (float)(f.factor * sin(a));
}

// ------------------------------------------------------------------- the cache
// The largest of a unit's values as bits: for magnitudes the order of the bits is the
// order of the values, and infinities and NaN come out above every finite one.
template <int LPU>
__device__ __forceinline__ unsigned unit_max(unsigned v) {
#pragma unroll
  for (int m = LPU / 2; m >= 1; m >>= 1) v = max(v, (unsigned)__shfl_xor((int)v, m));
  return v;
}

// 128 + the integer nearest to 127 x / top, ties to even, exactly: the fp32 quotient t is
// within 2^-15 of it, so only a t next to a border is decided again, by comparing
// 254 |x| with (2 m + 1) top, both of which 53 bits hold.
__device__ __forceinline__ unsigned code_of(float x, float top, float inv) {
  const float u = fabsf(x) * inv;
  const float m = floorf(u);
  float k = rintf(u);
  if (fabsf((u - m) - 0.5f) < 1e-4f) {
    const double l = 254.0 * (double)fabsf(x), r = (2.0 * (double)m + 1.0) * (double)top;
    k = l > r ? m + 1.f : l < r ? m : m + (float)((int)m & 1);
  }
  return 128u + (unsigned)(int)copysignf(k, x);
}

// The eight codes of a lane (two words) and the unit's scale.
template <int LPU>
__device__ __forceinline__ float quantise(const float (&x)[8], unsigned (&w)[2]) {
  unsigned b = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) b = max(b, __float_as_uint(x[i]) & 0x7fffffffu);
  b = unit_max<LPU>(b);
  w[0] = w[1] = 0x80808080u;
  // a row holding an infinity or a NaN is kept as NaN, so that what reads it shows it
  if (b >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
  const float top = fmaxf(__uint_as_float(b), kKv8Least), inv = __fdiv_rn(127.f, top);
  unsigned q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = code_of(x[i], top, inv);
  w[0] = q[0] | q[1] << 8 | q[2] << 16 | q[3] << 24;
  w[1] = q[4] | q[5] << 8 | q[6] << 16 | q[7] << 24;
  return __fdiv_rn(top, 127.f);
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
// The block of a position's page, or nullptr when no page holds it.
template <int HD>
__device__ __forceinline__ char* block_of(const Kv8& c, const RowAt& w, int which, int h) {
  if (!w.there) return nullptr;
  const int phys = kv8_page(w.table, w.pos >> c.page_shift, c.max_pages, c.n_pages);
  return phys < 0 ? nullptr
                  : w.base + kv8_block_at(phys, which, h, c.n_kv, 1 << c.page_shift, HD);
}
// Whether R rows are the R positions of one word of value codes (in a page that exists).
template <int R>
__device__ __forceinline__ bool one_word(const RowAt (&w)[R], char* const (&blk)[R]) {
  return R == 4 && blk[0] && (w[0].pos & 3) == 0 && w[R - 1].there && w[R - 1].end == w[0].end &&
         w[R - 1].table == w[0].table && w[R - 1].pos == w[0].pos + R - 1;
}

// A unit takes R neighbouring rows of one head.  The rows do not wait for their places, so
// they are requested first.  With four rows (prompts) a value word of four positions is
// written whole where the rows are those four: single bytes took 14.7 us for 2048 rows of 8
// heads of 128, now 11: 8.4 MB in and 4.3 out, of which a call of 48 rows already takes the
// first 4.7 (a row's place is three loads, one after another).  What bounds it is not known:
// neither bytes (2.4 us) nor arithmetic nor that chain, since half the vector instructions, or one
// load less in the chain, changed nothing.
// 12 prompts of up to 500 rows whose positions start anywhere in a word (fp32, heads of 64)
// take 15 us, their values written byte by byte.
template <int HD, int R>
__global__ __launch_bounds__(256) void k_kv8_append(Kv8 c, Kv8Rows r, RopeTab rope, int n_q,
                                                    HeadRows q, HeadRows q_out, float q_scale,
                                                    HeadRows k, HeadRows v) {
  constexpr int LPU = HD / 8, UPB = 256 / LPU;
  const int lane = threadIdx.x % LPU, per = n_q + 2 * c.n_kv;
  const unsigned u = blockIdx.x * UPB + threadIdx.x / LPU;  // below 2^28
  const int t = R * (int)(u / per), item = (int)(u % per);
  if (t >= r.n_rows) return;  // whole units leave together
  const bool is_q = item < n_q, is_v = item >= n_q + c.n_kv;
  const int h = is_q ? item : is_v ? item - n_q - c.n_kv : item - n_q;
  const HeadRows& x = is_q ? q : is_v ? v : k;
  RopeTab none = rope;
  none.cos = nullptr;
  const Runs run = runs(is_v ? none : rope, lane);
  float e[R][8];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int64_t in = min(t + i, r.n_rows - 1) * x.row_stride + h * x.head_stride;
    load44(x, in, run.a, run.b, e[i]);
    for (int s = 1; s < x.n_sum; ++s) {
      float m[8];
      load4(x, in + s * x.sum_stride + run.a, m);
      load4(x, in + s * x.sum_stride + run.b, m + 4);
#pragma unroll
      for (int j = 0; j < 8; ++j) e[i][j] += m[j];
    }
  }
  RowAt w[R];
  rows_at<LPU>(w, c, r, t, lane);
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (w[i].there) turn_row(rope, run, lane, w[i].pos, e[i]);
  if (is_q) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (!w[i].there) continue;
#pragma unroll
      for (int j = 0; j < 8; ++j) e[i][j] *= q_scale;
      put44(q_out, (t + i) * q_out.row_stride + h * q_out.head_stride, run.a, run.b, e[i]);
    }
    return;
  }
  const int page = 1 << c.page_shift;
  char* blk[R];
  unsigned code[R][2];
  float scale[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    blk[i] = block_of<HD>(c, w[i], is_v, h);
    scale[i] = quantise<LPU>(e[i], code[i]);
  }
  const int slot = w[0].pos & (page - 1);
  const bool word = one_word(w, blk);
  if (is_v && word) {
    unsigned d[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      d[j] = 0;
#pragma unroll
      for (int i = 0; i < R; ++i) d[j] |= (code[i][j >> 2] >> (8 * (j & 3)) & 0xffu) << (8 * (i & 3));
    }
    uint4* to = reinterpret_cast<uint4*>(blk[0] + kv8_value_at(slot, 8 * lane, HD));
    to[0] = make_uint4(d[0], d[1], d[2], d[3]);
    to[1] = make_uint4(d[4], d[5], d[6], d[7]);
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (!blk[i]) continue;
    const int at = w[i].pos & (page - 1);
    if (!is_v) {
      *reinterpret_cast<unsigned*>(blk[i] + kv8_key_at(at, run.a, HD)) = code[i][0];
      *reinterpret_cast<unsigned*>(blk[i] + kv8_key_at(at, run.b, HD)) = code[i][1];
    } else if (!word) {
      char* d = blk[i] + kv8_value_at(at, 8 * lane, HD);
#pragma unroll
      for (int j = 0; j < 8; ++j) d[4 * j] = (char)(code[i][j >> 2] >> (8 * (j & 3)));
    }
    if (lane == 0) *reinterpret_cast<float*>(blk[i] + kv8_scale_at(at, page, HD)) = scale[i];
  }
}

// Bound by memory where there is much to read: 16384 rows of 8 heads of 128 (to bf16) 22 us for
// 102 MB, 4.5 TB/s; 2048 rows 9 us.
template <int HD, int R>
__global__ __launch_bounds__(256) void k_kv8_read(Kv8 c, Kv8Rows r, HeadRows k, HeadRows v) {
  constexpr int LPU = HD / 8, UPB = 256 / LPU;
  const int lane = threadIdx.x % LPU, per = 2 * c.n_kv;
  const unsigned u = blockIdx.x * UPB + threadIdx.x / LPU;  // below 2^28
  const int t = R * (int)(u / per), item = (int)(u % per);
  if (t >= r.n_rows) return;
  RowAt w[R];
  rows_at<LPU>(w, c, r, t, lane);
  const bool is_v = item >= c.n_kv;
  const int h = is_v ? item - c.n_kv : item;
  const HeadRows& y = is_v ? v : k;
  if (!y.p) return;
  const int page = 1 << c.page_shift;
  char* blk[R];
#pragma unroll
  for (int i = 0; i < R; ++i) blk[i] = block_of<HD>(c, w[i], is_v, h);
  unsigned word[8];
  const bool one = is_v && one_word(w, blk);
  auto words = [&](const char* b, int at) {  // the value words of slot `at`
    const uint4* s = reinterpret_cast<const uint4*>(b + kv8_value_at(at & ~3, 8 * lane, HD));
    const uint4 x = s[0], z = s[1];
    word[0] = x.x; word[1] = x.y; word[2] = x.z; word[3] = x.w;
    word[4] = z.x; word[5] = z.y; word[6] = z.z; word[7] = z.w;
  };
  if (one) words(blk[0], w[0].pos & (page - 1));
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (!w[i].there) continue;
    float e[8] = {};  // a position without a page reads as zero
    if (blk[i]) {
      const int at = w[i].pos & (page - 1);
      const float scale = *reinterpret_cast<const float*>(blk[i] + kv8_scale_at(at, page, HD));
      unsigned code[8];
      if (is_v) {
        if (!one) words(blk[i], at);
#pragma unroll
        for (int j = 0; j < 8; ++j) code[j] = word[j] >> (8 * (at & 3)) & 0xffu;
      } else {
        const uint2 a = *reinterpret_cast<const uint2*>(blk[i] + kv8_key_at(at, 8 * lane, HD));
#pragma unroll
        for (int j = 0; j < 8; ++j) code[j] = (j < 4 ? a.x : a.y) >> (8 * (j & 3)) & 0xffu;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) e[j] = (float)((int)code[j] - 128) * scale;
    }
    put44(y, (t + i) * y.row_stride + h * y.head_stride, 8 * lane, 8 * lane + 4, e);
  }
}

// ------------------------------------------------------------------- launchers
// Workgroups of `units` units, or 0 when there are none or 2^28 and more (16 threads each, of
// 2^32 in a grid).
static unsigned unit_blocks(int hd, int64_t units) {
  const int64_t per = 256 / (hd / 8), n = (units + per - 1) / per;
  return units < 1 || units >= (int64_t)1 << 28 ? 0 : (unsigned)n;
}

hipError_t launch_rope_rows(int hd, const HeadRows& x, const HeadRows& y, int n_rows, int n_heads,
                            const int32_t* positions, const RopeTab& rope, hipStream_t st) {
  const bool halves = rope.layout == 0 && rope.dim % 16 == 0 && x.bf16 && y.bf16;
  // (the second, of half as many lanes a unit, in as many fewer workgroups)
  const unsigned full = unit_blocks(hd, (int64_t)n_rows * n_heads), grid = halves ? (full + 1) / 2 : full;
  if (!full) return hipErrorInvalidValue;
#define WICI_ROPE(K)                                                                          \
  launch_k(K, dim3(grid), dim3(256), 0, st, kOnly, x, y, n_rows, n_heads, positions, rope)
  if (hd == 128 && halves) WICI_ROPE(k_rope_halves<128>);
  else if (hd == 128) WICI_ROPE(k_rope_rows<128>);
  else if (hd == 64 && halves) WICI_ROPE(k_rope_halves<64>);
  else if (hd == 64) WICI_ROPE(k_rope_rows<64>);
  else return hipErrorInvalidValue;
#undef WICI_ROPE
  return hipGetLastError();
}

hipError_t launch_rope_table(const RopeFreqs& f, int half, int64_t n_pos, float* cos, float* sin,
                             hipStream_t st) {
  const int64_t n = n_pos * half, grid = (n + 255) / 256;
  if (half < 1 || half > 64 || grid < 1 || grid > 0x7fffffff) return hipErrorInvalidValue;
  launch_k(k_rope_table, dim3((unsigned)grid), dim3(256), 0, st, kOnly, f, half, n, cos, sin);
  return hipGetLastError();
}

// Rows a unit takes: four of a prompt, one where rows are few or belong to as many sequences.
static int rows_of_unit(const Kv8Rows& r) { return r.n_rows >= 64 && r.n_rows >= 4 * r.n_seqs ? 4 : 1; }

hipError_t launch_kv8_append(int hd, const Kv8& c, const Kv8Rows& r, const RopeTab& rope, int n_q,
                             const HeadRows& q, const HeadRows& q_out, float q_scale,
                             const HeadRows& k, const HeadRows& v, hipStream_t st, int edge) {
  if (!q.p) n_q = 0;
  const int R = rows_of_unit(r);
  const unsigned grid = unit_blocks(hd, ((int64_t)r.n_rows + R - 1) / R * (n_q + 2 * c.n_kv));
  if (!grid) return hipErrorInvalidValue;
#define WICI_APPEND(HD, R)                                                                       \
  launch_k(k_kv8_append<HD, R>, dim3(grid), dim3(256), 0, st, edge, c, r, rope, n_q, q, q_out, \
           q_scale, k, v)
  if (hd == 128 && R == 4) WICI_APPEND(128, 4);
  else if (hd == 128) WICI_APPEND(128, 1);
  else if (hd == 64 && R == 4) WICI_APPEND(64, 4);
  else if (hd == 64) WICI_APPEND(64, 1);
  else return hipErrorInvalidValue;
#undef WICI_APPEND
  return hipGetLastError();
}

hipError_t launch_kv8_read(int hd, const Kv8& c, const Kv8Rows& r, const HeadRows& k,
                           const HeadRows& v, hipStream_t st) {
  const int R = rows_of_unit(r);
  const unsigned grid = unit_blocks(hd, ((int64_t)r.n_rows + R - 1) / R * 2 * c.n_kv);
  if (!grid) return hipErrorInvalidValue;
#define WICI_READ(HD, R) \
  launch_k(k_kv8_read<HD, R>, dim3(grid), dim3(256), 0, st, kOnly, c, r, k, v)
  if (hd == 128 && R == 4) WICI_READ(128, 4);
  else if (hd == 128) WICI_READ(128, 1);
  else if (hd == 64 && R == 4) WICI_READ(64, 4);
  else if (hd == 64) WICI_READ(64, 1);
  else return hipErrorInvalidValue;
#undef WICI_READ
  return hipGetLastError();
}

}  // namespace wici
