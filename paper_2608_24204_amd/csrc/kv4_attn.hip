// Causal grouped-query attention over the 4-bit key-value cache.
//
// Mathematics.  For a row with query q over positions j with key rows k_j and value rows v_j:
//   y_j = (q . k_j) scale log2(e),   out = sum_j 2^(y_j - ref) v_j / sum_j 2^(y_j - ref),
// `ref` running with the largest y_j (an online softmax): it moves only when weights outgrow the size
// at which it was set (Room).  A cached value is one of 8 small numbers times a power of two, exact in
// bf16 over fp32's whole range: one conversion instruction makes two operands of a byte and a scale,
// and the scales need no arithmetic of their own.  The keys' product runs on the bf16 matrix cores,
// with the query as NQ bf16 terms: one for bf16 rows (exact), else three (2^-24).  Weights and values of
// bf16 rows enter the second product as one fp16 term while the values' scales are 2^-23 .. 2^8, so
// that fp16 holds them exactly (a weight to 2^-11, an eighth of the output's own rounding, or to 2^-31
// of the row's largest); where they are not, and for other rows, as NW bf16 terms (two, 2^-16, or
// three, 2^-24).  A wavefront that has met such a step goes on in bf16; groups of zeros, whose scale is
// the least, do that too (2048 rows of 8192 positions 366 us for 280).  Scores, weights, sums and the
// output are fp32.
//
// (The matrix instruction that takes 4-bit operands with their scales as they lie would need queries
// in 8 bits, two terms for bf16 ones at the same rate, and was measured to keep only about 2^-14 of the
// largest product in its sums of 32.)
//
// A value row that is NaN (scale bytes 255) must not reach rows that do not see it, and a product
// with a weight of zero would: its operands are made with another scale, and the weights of the
// rows that do see it are NaN instead.
//
// Layout.  S^T = K Q^T and O^T = V^T W^T on 16x16x32 products, as over the 8-bit cache: lane l holds
// query row l % 16 in both results, a tile of S^T leaves it with positions 4 (l / 16) .. + 3, and those
// are the positions that the second product takes from it.  For the keys a lane takes position l % 16
// and a quarter of the dimensions, within one group's scale; for the values four positions of hd / 16
// neighbouring dimensions, and their four scales.
#include <algorithm>
#include <type_traits>

#include "kv4.h"
#include "kv4_plan.h"
#include "kv_attn.h"
#include "launch.h"

namespace wici {

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
template <typename T> struct ElemOf;
template <> struct ElemOf<bf16x8_t> { typedef __bf16 type; };
template <> struct ElemOf<half8_t> { typedef _Float16 type; };
template <typename T> using Elem_t = typename ElemOf<T>::type;

// The state of 16 query rows over the positions a wavefront has taken: lane l, row l % 16.
struct RowState4 {
  float ref = kNoRef, sum = 0.f;  // sum over this lane's positions
};
// Output of 16 rows: tile u, element i: dimension (HD / 16) (4 (l / 16) + i) + u.
template <int HD>
using RowOut4 = floatx4_t[HD / 16];

// Byte i of a word of scales as the power of two that the conversions take: they read the exponent's
// bits alone (checked for every scale), so that what else the word holds may stand beside them.
__device__ __forceinline__ float scale_of(unsigned w, int i) {
  return __uint_as_float(i < 3 ? w << (23 - 8 * i) : w >> 1);
}
template <int BYTE>
__device__ __forceinline__ unsigned pair_of(unsigned w, float scale) {
  return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, BYTE));
}
// A word of key codes, eight dimensions of a position, as an operand.
__device__ __forceinline__ bf16x8_t keys8(unsigned w, float scale) {
  return __builtin_bit_cast(bf16x8_t, make_uint4(pair_of<0>(w, scale), pair_of<1>(w, scale),
                                                 pair_of<2>(w, scale), pair_of<3>(w, scale)));
}
// A word of value codes, four positions of a pair of dimensions: the positions of the first
// dimension (lo) and of the second, as bf16 or fp16.
template <int BYTE, bool HALF>
__device__ __forceinline__ unsigned pair_as(unsigned w, float scale) {
  if constexpr (HALF)
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, BYTE));
  else
    return pair_of<BYTE>(w, scale);
}
template <bool HALF>
__device__ __forceinline__ void values4(unsigned w, const float (&s)[4], uint2& lo, uint2& hi) {
  const unsigned a = pair_as<0, HALF>(w, s[0]), b = pair_as<1, HALF>(w, s[1]),
                 c = pair_as<2, HALF>(w, s[2]), d = pair_as<3, HALF>(w, s[3]);
  lo = make_uint2(__builtin_amdgcn_perm(b, a, 0x05040100u), __builtin_amdgcn_perm(d, c, 0x05040100u));
  hi = make_uint2(__builtin_amdgcn_perm(b, a, 0x07060302u), __builtin_amdgcn_perm(d, c, 0x07060302u));
}
// Which of a word's four positions are NaN (scale byte 255; 253 and 254, which memory never
// appended to may hold, are taken as it: 4 times theirs is infinite), as bits; their scales become 1.
// `large`: whether the wavefront has a scale that is large for rows of n positions (asked where LARGE: one
// that fits halves is not; asked everywhere, 2048 rows of 8192 positions took 286 us for 282).
template <bool LARGE>
__device__ __forceinline__ unsigned take_nans(unsigned& w, bool& large, const Room& room, int n) {
  const bool maybe = (w & w << 1 & 0x80808080u) != 0;  // some scale of 2^65 and more
  unsigned nan = 0;
  if (__builtin_expect(__any(maybe), false)) {
    bool big = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned byte = w >> (8 * i) & 0xffu;
      if (byte > (unsigned)kKv4MostByte) {
        nan |= 1u << i;
        w = (w & ~(0xffu << (8 * i))) | 127u << (8 * i);
      } else if constexpr (LARGE) {
        big |= byte >= (unsigned)kv4_large_byte(room, n);
      }
    }
    if constexpr (LARGE) large |= __any(big);
  }
  return nan;
}

// Whether one of a word's scales is outside 2^-23 .. 2^8 (bytes 104 .. 135), where fp16 holds
// every multiple of them.  (A byte of 232 and more carries into the next, and is outside itself.)
__device__ __forceinline__ bool past_half(unsigned w) {
  return ((w + 0x18181818u) & 0xe0e0e0e0u) != 0x80808080u;
}
// A word's scales from position `left` on become 1, or all where the page is absent: what nobody
// sees is finite in the products, and no result depends on it.
__device__ __forceinline__ void leave_seen(unsigned& w, bool there, int left) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (!there || i >= left) w = (w & ~(0xffu << (8 * i))) | 127u << (8 * i);
}

// The codes and scales of a step, as one lane holds them.
template <int HD>
struct Step4 {
  unsigned k[kTiles][HD / 32], ks[kTiles];  // position l % 16, dimensions (HD / 4) (l / 16) ..
  unsigned v[kTiles][HD / 32], vs[kTiles];  // positions 4 (l / 16) .. + 3, dimensions (HD / 16) (l % 16) ..
};
// (ONCE: not kept in the caches.)
template <bool ONCE = false, int N>
__device__ __forceinline__ void fetch_words(unsigned (&w)[N], __amdgpu_buffer_rsrc_t r, int lane_at,
                                            int at) {
  constexpr int kNonTemporal = ONCE ? 2 : 0;
  if constexpr (N == 4) {
    const u32x4_t v = __builtin_amdgcn_raw_buffer_load_b128(r, lane_at, at, kNonTemporal);
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
  } else if constexpr (N == 2) {
    const auto v = __builtin_amdgcn_raw_buffer_load_b64(r, lane_at, at, kNonTemporal);
    w[0] = v[0]; w[1] = v[1];
  } else {
    w[0] = __builtin_amdgcn_raw_buffer_load_b32(r, lane_at, at, kNonTemporal);
  }
}
// One KV head of a pool: its key block in page 0, and the bytes from page to page and from a
// key block to its value block.
template <int HD>
struct HeadAt4 {
  const char* base;
  uint32_t page, values;
  __device__ __forceinline__ HeadAt4(const Kv8& c, const Kv8Seq& q, int h)
      : base(q.base + kv4_block_at(0, 0, h, c.n_kv, 1 << c.page_shift, HD)),
        page(2 * c.n_kv * (uint32_t)kv4_block_bytes(1 << c.page_shift, HD)),
        values(page / 2) {}
  // (on: false reads as zeros, from no memory)
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const Kv8& c, int phys, int which,
                                                           bool on = true) const {
    return rsrc(base + (uint64_t)(uint32_t)max(phys, 0) * page + (which ? values : 0),
                on ? kv4_block_bytes(1 << c.page_shift, HD) : 0);
  }
};
template <int HD, bool ONCE>
__device__ __forceinline__ void load_keys4(Step4<HD>& s, const Kv8& c, const HeadAt4<HD>& at,
                                           const Pages& p, int step, int lane, bool on) {
  const int page = 1 << c.page_shift, pos = lane & 15, d = (lane >> 4) * (HD / 4);
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const int slot = (int)(((uint32_t)step * kStep + 16 * t) & (uint32_t)(page - 1));
    const __amdgpu_buffer_rsrc_t b = at.buffer(c, p.phys[t], 0, on);
    fetch_words<ONCE>(s.k[t], b, kv4_key_at(pos, d, HD), kv4_key_at(slot, 0, HD));
    s.ks[t] = __builtin_amdgcn_raw_buffer_load_b8(b, pos * (HD / kKv4Group) + d / kKv4Group,
                                                  kv4_key_scale_at(slot, 0, page, HD), 0);
  }
}
template <int HD, bool ONCE>
__device__ __forceinline__ void load_values4(Step4<HD>& s, const Kv8& c, const HeadAt4<HD>& at,
                                             const Pages& p, int step, int lane) {
  const int page = 1 << c.page_shift, pos = 4 * (lane >> 4), d = (lane & 15) * (HD / 16);
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const int slot = (int)(((uint32_t)step * kStep + 16 * t) & (uint32_t)(page - 1));
    const __amdgpu_buffer_rsrc_t b = at.buffer(c, p.phys[t], 1);
    fetch_words<ONCE>(s.v[t], b, kv4_value_at(pos, d, HD), kv4_value_at(slot, 0, HD));
    s.vs[t] = __builtin_amdgcn_raw_buffer_load_b32(b, pos * (HD / kKv4Group) + 4 * (d / kKv4Group),
                                                   kv4_value_scale_at(slot, 0, page, HD), 0);
  }
}

__device__ __forceinline__ floatx4_t product(bf16x8_t a, bf16x8_t b, floatx4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ floatx4_t product(half8_t a, half8_t b, floatx4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// S^T of one step: sc[t][i] is the product of position 16 t + 4 (l / 16) + i with row l % 16.
template <int HD, int NQ>
__device__ __forceinline__ void scores4(floatx4_t (&sc)[kTiles], const Step4<HD>& s,
                                        const bf16x8_t (&qf)[NQ][HD / 32]) {
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const float scale = __uint_as_float(s.ks[t] << 23);
    sc[t] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) {
      const bf16x8_t a = keys8(s.k[t][d], scale);
#pragma unroll
      for (int n = 0; n < NQ; ++n)
        sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[n][d], sc[t], 0, 0, 0);
    }
  }
}

// The weights of 32 positions from their products (a score is product * unit), as NW terms of type
// T.  MASKED: some row does not see every position: row l % 16 sees those below `seen`, of the tiles
// that are there.  nan: the positions (bit 4 t + i) whose weight is NaN.  The terms are those of 2^-lift
// of the weights (the same in the wavefront; 0 for halves).  Returns whether a row's reference moved:
// the output so far is then to be multiplied by `corr`.
//
// What is rare stands in one branch: NaN values, a reference to move (once a lane's eight weights
// sum up to more than room.most: one comparison), and references past 2^22 (`huge`: one of these 16
// rows has such a one).  From those a product is subtracted after it is rounded, as it was for the reference:
// joined, the difference of scores that are equal and that large would not be zero.  A row's weights
// are made of its own values alone, whatever takes the wavefront into the branch.
template <typename T, int NW, bool MASKED>
__device__ __forceinline__ bool weights4(T (&wf)[NW], RowState4& st, bool& huge,
                                         const floatx4_t (&sc)[kTiles], const Pages& p, float unit,
                                         unsigned nan, const Room& room, float lift, int seen,
                                         int lane, float& corr) {
  const int left = MASKED ? fresh(seen - 4 * (lane >> 4)) : 0;
  auto on = [&](int t, int i) { return !MASKED || (p.phys[t] >= 0 && 16 * t + i < left); };
  float w[4 * kTiles], sum;
  // d(t, i): a score less the reference
  auto weigh = [&](auto d) {
    sum = 0.f;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[4 * t + i] = __builtin_amdgcn_exp2f(on(t, i) ? d(t, i) : -INFINITY);
        sum += w[4 * t + i];
      }
  };
  weigh([&](int t, int i) { return __builtin_fmaf(sc[t][i], unit, -st.ref); });
  bool move = false;
  if (__builtin_expect(__any(!(sum <= room.most)) || huge || __any(nan != 0), false)) {
    // (made here, and not for every step ahead of the branch)
    const unsigned bits = (unsigned)fresh((int)nan);
    float x[4 * kTiles], y[4 * kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v = sc[t][i];
        asm volatile("" : "+v"(v));
        v = bits >> (4 * t + i) & 1 ? __uint_as_float(0x7fc00000u) : v;
        x[4 * t + i] = v;
        v *= unit;
        asm volatile("" : "+v"(v));
        y[4 * t + i] = v;
      }
    auto distance = [&](int t, int i) {
      const float d = y[4 * t + i] - st.ref;
      return fabsf(st.ref) > 0x1p22f ? d : __builtin_fmaf(x[4 * t + i], unit, -st.ref);
    };
    weigh(distance);
    const uint64_t lanes = __ballot(!(sum <= room.most));  // lanes l, l + 16, .. : row l
    if (lanes) {
      move = true;
      const uint32_t two = (uint32_t)lanes | (uint32_t)(lanes >> 32);
      const bool mine = (two | two >> 16) >> (lane & 15) & 1;
      float z = -INFINITY;
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (on(t, i)) z = fmaxf(z, y[4 * t + i]);
      z = fmaxf(z, __shfl_xor(z, 16));
      z = fmaxf(z, __shfl_xor(z, 32));
      const float ref = mine ? fmaxf(st.ref, z - room.top) : st.ref;
      corr = mine ? __builtin_amdgcn_exp2f(st.ref - ref) : 1.f;
      st.sum *= corr;
      st.ref = ref;
      huge = __any(fabsf(ref) > 0x1p22f && ref != kNoRef);
      weigh(distance);
    }
  }
  st.sum += sum;
  if constexpr (!std::is_same<T, half8_t>::value) {
    if (__builtin_expect(lift != 0.f, false)) {
      const float down = __builtin_amdgcn_exp2f(-lift);
#pragma unroll
      for (int i = 0; i < 4 * kTiles; ++i) w[i] *= down;
    }
  }
#pragma unroll
  for (int i = 0; i < 4 * kTiles; ++i) {
    float rest = w[i];
#pragma unroll
    for (int n = 0; n < NW; ++n) {
      wf[n][i] = (Elem_t<T>)rest;
      rest -= (float)wf[n][i];
    }
  }
  return move;
}

// O^T += V^T W^T of one step; vs: the scales, NaN ones replaced.
template <int HD, typename T, int NW>
__device__ __forceinline__ void add_values4(RowOut4<HD>& o, const Step4<HD>& s,
                                            const unsigned (&vs)[kTiles], const T (&wf)[NW]) {
  constexpr bool kHalf = std::is_same<T, half8_t>::value;
  float f[kTiles][4];
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) f[t][i] = scale_of(vs[t], i);
#pragma unroll
  for (int d = 0; d < HD / 32; ++d) {
    uint2 a0, a1, b0, b1;
    values4<kHalf>(s.v[0][d], f[0], a0, b0);
    values4<kHalf>(s.v[1][d], f[1], a1, b1);
    const T a = __builtin_bit_cast(T, make_uint4(a0.x, a0.y, a1.x, a1.y));
    const T b = __builtin_bit_cast(T, make_uint4(b0.x, b0.y, b1.x, b1.y));
#pragma unroll
    for (int n = 0; n < NW; ++n) {
      o[2 * d] = product(a, wf[n], o[2 * d]);
      o[2 * d + 1] = product(b, wf[n], o[2 * d + 1]);
    }
  }
}

template <int HD>
__device__ __forceinline__ void rescale4(RowOut4<HD>& o, float f) {
#pragma unroll
  for (int u = 0; u < HD / 16; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[u][i] *= f;
}

// 16 query rows (row l % 16 of the tile, zero where `on` is false) as NQ bf16 terms.
template <int HD, int NQ>
__device__ __forceinline__ void load_queries4(const HeadRows& q, int64_t at, bool on, int lane,
                                              bf16x8_t (&qf)[NQ][HD / 32]) {
  at += (lane >> 4) * (HD / 4);
  if (NQ == 1 || q.bf16) {
    uint4 raw[HD / 32];
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
      raw[d] = *reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(q.p) + at + 8 * d);
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) {
      qf[0][d] = __builtin_bit_cast(bf16x8_t, on ? raw[d] : make_uint4(0, 0, 0, 0));
#pragma unroll
      for (int n = 1; n < NQ; ++n) qf[n][d] = bf16x8_t{};
    }
  } else {
    float v[HD / 32][8];
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) load8(static_cast<const float*>(q.p) + at + 8 * d, v[d]);
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float rest = on ? v[d][i] : 0.f;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          qf[n][d][i] = (__bf16)rest;
          rest -= (float)qf[n][d][i];
        }
      }
  }
}

// ------------------------------------------------------------------- split over positions
// Workgroup (KV head, sequence, split): four wavefronts take the split's steps of 32
// positions in turn for a tile of 16 of the sequence's rows x query heads of the group
// (row r: new row r / G, query head r % G), and are joined at the end.  Splits take
// groups of four steps in turn, so one launch serves any length evenly.  With one
// split the output is written here, otherwise (ref, sum, output) is left for the merge.
// ONCE: nobody reads a code again.
//
// Bound by the cache's bytes, each read once: 32 tokens at 16384 (40 query on 8 KV heads of 128, bf16)
// 93 us for 570 MB, 6.1 TB/s where a large copy moves 4.8-5.2; the loads with nothing behind them take
// 92.  There the vector units are busy 54% of the time (17 instructions of a tile's 70 make keys, 36
// values).  Where there is less to read, latencies show: 48 tokens at up to 4000 (heads of 64) 28.7 us
// for 81 MB, one at 16384 (fp32) 12.8 us for 18 MB.  Three wavefronts a SIMD for heads of 128 (two with
// three terms), four for heads of 64: one more changed nothing (114 for 112, 37.8 for 36.7 us), nor did
// steps of 64 positions (124 for 120, 37.0 for 37.0).
template <int HD, int NQ, int NW, bool ONCE>
__global__ __launch_bounds__(256)
__attribute__((amdgpu_waves_per_eu(HD == 64 ? 4 : NQ == 1 ? 3 : 2))) void k_kv4_attn_split(
    Kv8 c, Kv8Rows r, Kv8Attn a, int nsplit, int ntile) {
  __shared__ float s_o[4][16][HD + 4];
  __shared__ float s_ref[4][16], s_sum[4][16], s_lift[4];
  const int h = blockIdx.x % c.n_kv, split = blockIdx.x / c.n_kv % nsplit;
  const int tile0 = blockIdx.x / (c.n_kv * nsplit), b = blockIdx.y;
  const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int r16 = lane & 15, G = a.n_q / c.n_kv;
  const Kv8Seq q = uniform(kv8_seq(c, r, b));
  const int64_t cap = (int64_t)c.max_pages << c.page_shift;
  const size_t parts = (size_t)r.n_rows * a.n_q * nsplit;
  // the wavefront's first steps do not depend on the length, so that their pages are
  // looked up beside it
  const HeadAt4<HD> kv(c, q, h);
  const int s0 = 4 * split + wave;
  const Entries e0 = find(c, q, s0), e1 = find(c, q, s0 + 4 * nsplit);

  for (int tile = tile0; tile * 16 < q.rows * G; tile += ntile) {
    const int qr = 16 * tile + r16, row = qr / G, head = h * G + qr % G;
    const bool on = row < q.rows;
    const int rc = min(row, q.rows - 1);
    // a row sees the positions up to its own; the tile's last row sees the most
    const int last = min((16 * tile + 15) / G, q.rows - 1), first = 16 * tile / G;
    auto seen = [&](int rr) { return kv8_seen(q.len, q.rows, rr, cap); };
    const int limit = on ? seen(row) : 0, steps = kv8_steps(seen(last), kStep);
    // steps that all 16 rows see whole
    const int whole = 16 * tile + 15 < q.rows * G ? seen(first) / kStep : 0;

    // the next step's keys are requested once this one's are multiplied, its values
    // likewise, and its pages (which those addresses wait for) a step earlier
    const int stride = 4 * nsplit;
    int s = s0;
    bf16x8_t qf[NQ][HD / 32];
    load_queries4<HD, NQ>(a.q, (q.row0 + rc) * a.q.row_stride + head * a.q.head_stride, on, lane, qf);
    const float unit = a.scale * kLog2e;
    constexpr Room room = NQ > 1 ? kRoomBf16 : kRoomHalf;
    float lift = 0.f;
    bool huge = false;
    RowState4 st;
    RowOut4<HD> o;
#pragma unroll
    for (int u = 0; u < HD / 16; ++u) o[u] = floatx4_t{0.f, 0.f, 0.f, 0.f};
    if (s < steps) {
      Step4<HD> x;
      Pages now = named(c, e0), next;
      Entries later = e1;
      floatx4_t sc[kTiles];
      bool scored = false;  // this step's scores are made, and the next one's keys requested
      load_keys4<HD, ONCE>(x, c, kv, now, s, lane, true);
      load_values4<HD, ONCE>(x, c, kv, now, s, lane);
      // The steps from here on, with the values and weights as halves or as NW bf16 terms; returns
      // whether none is left: halves end before the first step whose values do not fit them.
      auto take = [&](auto halves) -> bool {
        typedef std::conditional_t<halves.value, half8_t, bf16x8_t> Value;
        constexpr int N = halves.value ? 1 : NW;
        for (;;) {
          const int then = s + stride;
          if (halves.value || !scored) {
            scores4<HD, NQ>(sc, x, qf);
            next = named(c, later);
            // (in any case: what follows would else wait for whatever may be requested here)
            load_keys4<HD, ONCE>(x, c, kv, next, then, lane, then < steps);
          }
          scored = false;
          const bool clear = s < whole && now.all();
          unsigned vs[kTiles], nan = 0;
#pragma unroll
          for (int t = 0; t < kTiles; ++t) {
            vs[t] = x.vs[t];
            if (!clear)
              leave_seen(vs[t], now.phys[t] >= 0, seen(last) - s * kStep - (16 * t + 4 * (lane >> 4)));
          }
          if (!halves.value || __builtin_expect(__any(past_half(vs[0]) || past_half(vs[1])), false)) {
            bool large = false;
#pragma unroll
            for (int t = 0; t < kTiles; ++t) nan |= take_nans<!halves.value>(vs[t], large, room, seen(last)) << (4 * t);
            if (halves.value && __any(past_half(vs[0]) || past_half(vs[1]))) {
              scored = true;
              return false;
            }
            if (__builtin_expect(large, false) && lift == 0.f) {
              lift = (float)kv4_lift(room, seen(last));
              rescale4<HD>(o, __builtin_amdgcn_exp2f(-lift));
            }
          }
          Value wf[N];
          float corr = 1.f;
          const bool move =
              clear ? weights4<Value, N, false>(wf, st, huge, sc, now, unit, nan, room, lift, 0, lane, corr)
                    : weights4<Value, N, true>(wf, st, huge, sc, now, unit, nan, room, lift,
                                               limit - s * kStep, lane, corr);
          if (__builtin_expect(move, false)) rescale4<HD>(o, corr);
          add_values4<HD>(o, x, vs, wf);
          if (then >= steps) return true;
          load_values4<HD, ONCE>(x, c, kv, next, then, lane);
          now = next;
          later = find(c, q, then + stride);
          s = then;
        }
      };
      if (NQ > 1 || __builtin_expect(!take(std::integral_constant<bool, true>()), false))
        take(std::integral_constant<bool, false>());
    }
    // join the wavefronts
    st.sum += __shfl_xor(st.sum, 16);
    st.sum += __shfl_xor(st.sum, 32);
    note_no_weight(st.ref, st.sum, c, q, limit, s0 * kStep, seen(last), lane);
    const int me = fresh(lane), mr = me & 15, mg = me >> 4;
    if (mg == 0) {
      s_ref[wave][mr] = st.ref;
      s_sum[wave][mr] = st.sum;
    }
    if (lane == 0) s_lift[wave] = lift;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int u = 0; u < HD / 16; u += 4)
        *reinterpret_cast<float4*>(&s_o[wave][mr][HD / 16 * (4 * mg + i) + u]) =
            make_float4(o[u][i], o[u + 1][i], o[u + 2][i], o[u + 3][i]);
    __syncthreads();
    for (int x = fresh(threadIdx.x); x < 16 * HD / 4; x += 256) {
      const int rr = x / (HD / 4), d = 4 * (x % (HD / 4)), tr = 16 * tile + rr;
      if (tr >= q.rows * G) continue;
      float ref = s_ref[0][rr];
#pragma unroll
      for (int w = 1; w < 4; ++w) ref = fmaxf(ref, s_ref[w][rr]);
      float sum = 0.f, up = 0.f, all[4] = {};
      const bool lifts = s_lift[0] + s_lift[1] + s_lift[2] + s_lift[3] != 0.f;
      if (__builtin_expect(lifts, false)) {
        // the least with which no wavefront's output is multiplied by 2 or more
        up = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) up = fmaxf(up, s_lift[w] + (s_ref[w][rr] - ref));
        up = floorf(up);
      }
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        float f = __builtin_amdgcn_exp2f(s_ref[w][rr] - ref);
        const float4 v = *reinterpret_cast<const float4*>(&s_o[w][rr][d]);
        sum += f * s_sum[w][rr];
        if (__builtin_expect(lifts, false))
          f = __builtin_amdgcn_exp2f(s_ref[w][rr] - ref + (s_lift[w] - up));
        all[0] += f * v.x; all[1] += f * v.y; all[2] += f * v.z; all[3] += f * v.w;
      }
      leave(a, nsplit, split, parts, q.row0 + tr / G, h * G + tr % G, d, ref, up, sum, all);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------- prompts: row tiles
// Workgroup (KV head, tile of 64 or 128 rows x query heads, split, sequence): each of four
// wavefronts holds a quarter of the rows and takes every chunk of 64 positions of the split.  The
// codes of a chunk become operands once for all four, in LDS, lane by lane as the products read
// them (16 bytes a lane): a wavefront converts one of the four tiles.  Two buffers: the next chunk's
// codes are on their way while this one is multiplied, and one barrier a chunk parts a buffer's
// readers from its next writers.
//
// 2048 rows of 8192 positions (32 query on 8 KV heads of 128) take 280 us in bf16, 859 TFLOP/s of
// products where a large product reaches 1100-1300.  No unit is full: matrix cores 36%, vector units
// 43%, LDS 33% of the time (a seventh of that bank conflicts: a tile's values are written 8 bytes a
// lane); the two wavefronts a SIMD that the registers allow wait for each other's units and on LDS.  Two bf16 terms of every weight took 366 us; eight wavefronts of 16 rows a
// workgroup, four a SIMD, 346 (they spill); the next chunk's operands made between this one's two
// steps 289.
template <int HD, int NQ, int NW, int kRowTiles>
__global__ __launch_bounds__(256)
__attribute__((amdgpu_waves_per_eu(2))) void k_kv4_attn_tile(Kv8 c, Kv8Rows r, Kv8Attn a, int nsplit,
                                                            int ntile) {
  constexpr int DS = HD / 32, DT = HD / 16, kRows = 4 * 16 * kRowTiles;
  static_assert(kChunkTiles == 4, "a wavefront brings one tile of a chunk");
  enum Kind { kTooWide = 1, kNans = 2, kLarge = 4 };
  __shared__ uint4 s_k[2][kChunkTiles][DS][64];      // keys: tile, 32 dimensions, lane
  __shared__ uint4 s_v[2][kChunkTiles / 2][DT][64];  // values: two tiles, 16 dimensions, lane
  __shared__ __align__(16) int s_kind[2][kChunkTiles];         // of a tile's values: Kind,
  __shared__ unsigned s_nan[2][kChunkTiles][4];  // and which are NaN, by lane / 16
  const int h = blockIdx.x % c.n_kv, split = blockIdx.x / c.n_kv % nsplit;
  const int tile0 = blockIdx.x / (c.n_kv * nsplit), b = blockIdx.y;
  const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int r16 = lane & 15, g = lane >> 4, G = a.n_q / c.n_kv;
  const Kv8Seq q = uniform(kv8_seq(c, r, b));
  const int64_t cap = (int64_t)c.max_pages << c.page_shift;
  const int page = 1 << c.page_shift;
  const size_t parts = (size_t)r.n_rows * a.n_q * nsplit;
  const int total = q.rows * G, tiles = (total + kRows - 1) / kRows;
  const HeadAt4<HD> kv(c, q, h);
  const float unit = a.scale * kLog2e;
  const bool two_a_cu = gridDim.x > kCus && gridDim.x * gridDim.y <= 2 * kCus && tiles <= ntile;

  for (int back = tile0; back < tiles; back += ntile) {
    // From the last tile back; with two workgroups a CU, the second half from the first tile
    // on, so that a CU's two see about as many positions together as any other's.
    const int first = (tiles + 1) / 2;
    const int tile = two_a_cu && back >= first ? back - first : tiles - 1 - back;
    const int row0 = kRows * tile, mine = row0 + 16 * kRowTiles * wave;
    auto seen = [&](int rr) { return kv8_seen(q.len, q.rows, rr, cap); };
    // positions this wavefront's rows see at most and at least
    const int most = mine < total ? seen(min((mine + 16 * kRowTiles - 1) / G, q.rows - 1)) : 0;
    const int least = mine + 16 * kRowTiles <= total ? seen(mine / G) : 0;
    const int all = seen(min((row0 + kRows - 1) / G, q.rows - 1));  // of the workgroup's rows
    const int chunks = kv8_steps(all, kChunkPos), per = (chunks + nsplit - 1) / nsplit;
    const int c0 = min(split * per, chunks), c1 = min(c0 + per, chunks);

    RowState4 st[kRowTiles];
    RowOut4<HD> o[kRowTiles];
    constexpr Room room = NQ > 1 ? kRoomBf16 : kRoomHalf;
    float lift = 0.f;
    bool huge[kRowTiles];
#pragma unroll
    for (int x = 0; x < kRowTiles; ++x) {
      huge[x] = false;
#pragma unroll
      for (int u = 0; u < DT; ++u) o[x][u] = floatx4_t{0.f, 0.f, 0.f, 0.f};
    }

    // what this wavefront brings of a chunk: the keys and values of one tile
    unsigned kc[DS], ks, vc[DS], vs;
    int phys[kChunkTiles], later[kChunkTiles];
    const bool whole_chunk = c.page_shift >= 6;  // one page holds a chunk
    auto find = [&](int chunk) {
      later[0] = entry(c, q, (uint32_t)chunk * kChunkPos);
      if (!whole_chunk)
#pragma unroll
        for (int t = 1; t < kChunkTiles; ++t)
          later[t] = entry(c, q, (uint32_t)chunk * kChunkPos + 16 * t);
    };
    auto look = [&]() {
      phys[0] = kv8_named(later[0], c.n_pages);
#pragma unroll
      for (int t = 1; t < kChunkTiles; ++t)
        phys[t] = whole_chunk ? phys[0] : kv8_named(later[t], c.n_pages);
    };
    // p[t], with bits: a choice between the elements would put them into memory
    auto pick = [](const int (&p)[kChunkTiles], int t) {
      const int lo = p[0] ^ ((p[0] ^ p[1]) & -(t & 1)), hi = p[2] ^ ((p[2] ^ p[3]) & -(t & 1));
      return lo ^ ((lo ^ hi) & -(t >> 1));
    };
    auto bring = [&](const int (&p)[kChunkTiles], int chunk) {
      const int j0 = chunk * kChunkPos;
      const int phys = whole_chunk ? p[0] : pick(p, wave), slot = (j0 + 16 * wave) & (page - 1);
      const __amdgpu_buffer_rsrc_t kb = kv.buffer(c, phys, 0), vb = kv.buffer(c, phys, 1);
      const int dk = g * (HD / 4), dv = r16 * (HD / 16);
      fetch_words(kc, kb, kv4_key_at(r16, dk, HD), kv4_key_at(slot, 0, HD));
      ks = __builtin_amdgcn_raw_buffer_load_b8(kb, r16 * (HD / kKv4Group) + dk / kKv4Group,
                                               kv4_key_scale_at(slot, 0, page, HD), 0);
      fetch_words(vc, vb, kv4_value_at(4 * g, dv, HD), kv4_value_at(slot, 0, HD));
      vs = __builtin_amdgcn_raw_buffer_load_b32(vb, 4 * g * (HD / kKv4Group) + 4 * (dv / kKv4Group),
                                                kv4_value_scale_at(slot, 0, page, HD), 0);
    };
    // The operands of the chunk that is here; whether the values' scales do for `halves`.
    auto convert = [&](int buf, int ch, const int (&now)[kChunkTiles], auto halves) {
      const float scale = __uint_as_float(ks << 23);
#pragma unroll
      for (int d = 0; d < DS; ++d)
        s_k[buf][wave][d][lane] = __builtin_bit_cast(uint4, keys8(kc[d], scale));
      // (in the last chunk, and in pages that are not there)
      const int left = all - ch * kChunkPos;
      const int there = pick(now, wave);
      if (left < kChunkPos || there < 0) leave_seen(vs, there >= 0, left - (16 * wave + 4 * g));
      int kind = 0;
      if (!halves.value || __builtin_expect(__any(past_half(vs)), false)) {
        bool large = false;
        const unsigned nan = take_nans<!halves.value>(vs, large, room, all);
        kind = (large ? kLarge : 0) | (__any(nan != 0) ? kNans : 0) |
               (halves.value && __any(past_half(vs)) ? kTooWide : 0);
        if (r16 == 0) s_nan[buf][wave][g] = nan;
      }
      float f[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = scale_of(vs, i);
#pragma unroll
      for (int d = 0; d < DS; ++d) {
        uint2 lo, hi;
        values4<halves.value>(vc[d], f, lo, hi);
        uint4* to = &s_v[buf][wave >> 1][2 * d][lane];
        reinterpret_cast<uint2*>(to)[wave & 1] = lo;
        reinterpret_cast<uint2*>(to + 64)[wave & 1] = hi;
      }
      if (lane == 0) s_kind[buf][wave] = kind;
    };

    bf16x8_t qf[kRowTiles][NQ][DS];
    int limit[kRowTiles];  // positions each row sees
#pragma unroll
    for (int x = 0; x < kRowTiles; ++x) {
      const int qr = mine + 16 * x + r16, row = qr / G, rc = min(row, q.rows - 1);
      const bool on = qr < total;
      limit[x] = on ? seen(row) : 0;
      load_queries4<HD, NQ>(a.q, (q.row0 + rc) * a.q.row_stride + (h * G + qr % G) * a.q.head_stride,
                            on, lane, qf[x]);
    }
    // The chunks from `from` on, with the values and weights as halves or as NW bf16 terms; returns
    // the first chunk that it does not take: one whose values do not fit halves.
    auto take = [&](int from, auto halves) -> int {
      typedef std::conditional_t<halves.value, half8_t, bf16x8_t> Value;
      constexpr int N = halves.value ? 1 : NW;
      if (from >= c1) return from;
      find(from);
      look();
      bring(phys, from);
      find(from + 1);
      for (int ch = from; ch < c1; ++ch) {
        const int buf = (ch - from) & 1;
        int now[kChunkTiles];
#pragma unroll
        for (int t = 0; t < kChunkTiles; ++t) now[t] = phys[t];
        look();
        find(ch + 2);
        convert(buf, ch, now, halves);
        if (ch + 1 < c1) bring(phys, ch + 1);
        __syncthreads();
        const int4 k4 = *reinterpret_cast<const int4*>(s_kind[buf]);
        const int kinds[2] = {uniform(k4.x | k4.y), uniform(k4.z | k4.w)};
        if (halves.value && __builtin_expect((kinds[0] | kinds[1]) & kTooWide, false)) return ch;
        if (ch * kChunkPos >= most) continue;  // past this wavefront's rows
#pragma unroll
        for (int p = 0; p < kChunkTiles / 2; ++p) {
          const int j0 = ch * kChunkPos + 32 * p;
          Pages pg;
#pragma unroll
          for (int t = 0; t < kTiles; ++t) pg.phys[t] = now[2 * p + t];
          unsigned nan = 0;
          if (__builtin_expect(kinds[p], false)) {
            if (kinds[p] & kNans)
#pragma unroll
              for (int t = 0; t < kTiles; ++t)
                if (uniform(s_kind[buf][2 * p + t]) & kNans) nan |= s_nan[buf][2 * p + t][g] << (4 * t);
            if (!halves.value && (kinds[p] & kLarge) && lift == 0.f) {
              lift = (float)kv4_lift(room, all);
#pragma unroll
              for (int y = 0; y < kRowTiles; ++y)
                rescale4<HD>(o[y], __builtin_amdgcn_exp2f(-lift));
            }
          }
          // Row tile after row tile: the matrix cores work on one's products while the vector
          // units turn the other's scores into weights.
          floatx4_t x[kRowTiles][kTiles];
          uint4 op[DT];
#pragma unroll
          for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int d = 0; d < DS; ++d) op[t * DS + d] = s_k[buf][2 * p + t][d][lane];
#pragma unroll
          for (int y = 0; y < kRowTiles; ++y)
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
              x[y][t] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int d = 0; d < DS; ++d)
#pragma unroll
                for (int n = 0; n < NQ; ++n)
                  x[y][t] = product(__builtin_bit_cast(bf16x8_t, op[t * DS + d]), qf[y][n][d], x[y][t]);
            }
#pragma unroll
          for (int u = 0; u < DT; ++u) op[u] = s_v[buf][p][u][lane];
          const bool whole = least - j0 >= kStep && pg.all();
#pragma unroll
          for (int y = 0; y < kRowTiles; ++y) {
            float corr = 1.f;
            Value wf[N];
            const bool move =
                whole ? weights4<Value, N, false>(wf, st[y], huge[y], x[y], pg, unit, nan, room, lift, 0,
                                                  lane, corr)
                      : weights4<Value, N, true>(wf, st[y], huge[y], x[y], pg, unit, nan, room, lift,
                                                 limit[y] - j0, lane, corr);
            if (__builtin_expect(move, false)) rescale4<HD>(o[y], corr);
#pragma unroll
            for (int u = 0; u < DT; ++u)
#pragma unroll
              for (int n = 0; n < N; ++n)
                o[y][u] = product(__builtin_bit_cast(Value, op[u]), wf[n], o[y][u]);
          }
        }
      }
      return c1;
    };
    int at = c0;
    if (NQ == 1) at = take(at, std::integral_constant<bool, true>());
    if (NQ > 1 || __builtin_expect(at < c1, false)) {
      __syncthreads();  // (what was made of this chunk is read no more)
      take(at, std::integral_constant<bool, false>());
    }
    __syncthreads();  // the buffers are free for the next tile
    const int me = fresh(lane), mg = me >> 4;
#pragma unroll
    for (int y = 0; y < kRowTiles; ++y) {
      st[y].sum += __shfl_xor(st[y].sum, 16);
      st[y].sum += __shfl_xor(st[y].sum, 32);
      note_no_weight(st[y].ref, st[y].sum, c, q, limit[y], (uint32_t)c0 * kChunkPos, most, lane);
      const int qr = mine + 16 * y + (me & 15);
      if (qr >= total) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int u = 0; u < DT; u += 4) {
          float v[4] = {o[y][u][i], o[y][u + 1][i], o[y][u + 2][i], o[y][u + 3][i]};
          leave(a, nsplit, split, parts, q.row0 + qr / G, h * G + qr % G,
                DT * (4 * mg + i) + u, st[y].ref, lift, st[y].sum, v);
        }
    }
  }
}

// ------------------------------------------------------------------- launcher
size_t kv4_attn_floats(int hd, int n_q, int n_kv, int n_seqs, int n_rows, int max_rows,
                       int max_length) {
  const Kv8Plan p = kv4_plan(hd, 1, n_q, n_kv, n_seqs, max_rows, max_length);
  return p.nsplit == 1 ? 0 : kv8_part_floats((size_t)n_rows * n_q * p.nsplit, hd);
}

template <int HD>
static hipError_t attn4(const Kv8& c, const Kv8Rows& r, const Kv8Attn& a, hipStream_t st, int last) {
  // bf16 queries and output: one term of the query, one or two of the weights; else three
  const bool single = a.q.bf16 && a.out.p && a.out.bf16;
  const Kv8Plan p = kv4_plan(HD, single ? 1 : 3, a.n_q, c.n_kv, r.n_seqs, a.max_rows, a.max_length);
  const int64_t gx = (int64_t)c.n_kv * p.nsplit * p.ntile;
  if (gx > 0x7fffffff || r.n_seqs > 65535 || (p.nsplit > 1 && !a.work)) return hipErrorInvalidValue;
  const dim3 grid((unsigned)gx, r.n_seqs);
  const int edge = p.nsplit == 1 ? last : last & kFirst;
#define WICI_ATTN(...) \
  launch_k((__VA_ARGS__), grid, dim3(256), 0, st, edge, c, r, a, p.nsplit, p.ntile)
  if (p.row_tiles == 2) {
    WICI_ATTN(k_kv4_attn_tile<HD, 1, 2, 2>);
  } else if (p.row_tiles == 1) {
    if (single) WICI_ATTN(k_kv4_attn_tile<HD, 1, 2, 1>);
    else WICI_ATTN(k_kv4_attn_tile<HD, 3, 3, 1>);
  } else {
    // Codes that one tile of rows reads are read past the caches (heads of 128: 48 tokens at up to
    // 4000 positions 42.4 us for 46.0, 32 at 16384 103.6 for 119; heads of 64: 34.4 for 32.6, so
    // not there; 4 x 16 rows, four tiles, of 8000 31.9 for 29.9).
    constexpr bool kMay = HD == 128;
    if (kMay && p.ntile == 1) {
      if (single) WICI_ATTN(k_kv4_attn_split<HD, 1, 2, kMay>);
      else WICI_ATTN(k_kv4_attn_split<HD, 3, 3, kMay>);
    } else {
      if (single) WICI_ATTN(k_kv4_attn_split<HD, 1, 2, false>);
      else WICI_ATTN(k_kv4_attn_split<HD, 3, 3, false>);
    }
  }
#undef WICI_ATTN
  if (p.nsplit > 1) return launch_kv_attn_merge(HD, c, r, a, p.nsplit, st, last & kLast);
  return hipGetLastError();
}

hipError_t launch_kv4_attn(const Kv8& c, const Kv8Rows& r, const Kv8Attn& a, hipStream_t st,
                           int edge) {
  if (a.hd == 128) return attn4<128>(c, r, a, st, edge);
  if (a.hd == 64) return attn4<64>(c, r, a, st, edge);
  return hipErrorInvalidValue;
}

}  // namespace wici
