// Causal grouped-query attention over the 8-bit key-value cache.
//
// Mathematics.  For a row with query q over positions j with key codes a_j (scale s_j)
// and value codes c_j (scale t_j):
//   y_j = s_j (q . a_j) scale log2(e),   out = sum_j 2^y_j t_j c_j / sum_j 2^y_j.
// The codes are small integers, exact in fp16, so both products run on the fp16 matrix
// cores with the scales outside them: the keys' on the scores, the values' on the
// weights w_j = 2^(y_j - ref) t_j.  `ref` runs with the largest y_j + log2 t_j (an online
// softmax on the weights themselves), so the weights stay inside fp16's range, and one
// factor 2^-ref cancels in the quotient.  It moves only when a weight would pass 2^15 (it is
// set 2^6 below the largest), so most steps rescale nothing.  That one reference serves the
// sum too while it is near the largest score: values' scales are 2^-67 (a row of zeros) and
// more, and up to scales of 2^20 a sum of 2^(y_j - ref) is between 2^-14 and 2^83 of a term
// at the largest score, so that neither it nor the factors between two references leave
// fp32.  Where a scale is larger, or a score passes 2^24 (a reference then cannot hold log2 t_j
// beside it), rows go on with the largest score as `ref` and a power of two of the outputs'
// own, `lift`: they hold 2^-lift of their sum (`apart` below).  Scores,
// weights, sums and the output are fp32; q and w enter the products as NT fp16 terms: one
// for bf16 rows (q is exact in it, a weight within 2^-11, an eighth of the output's own
// rounding), two where queries or output are fp32 (2^-22); a weight 2^-20 and more below
// the largest, within 2^-31 of that.
//
// Layout.  S^T = A Q^T and O^T = C^T W^T on v_mfma_f32_16x16x32_f16: lane l holds query
// row l % 16 in both results, so maximum, sum and rescaling of a row are that lane's own
// (lanes l, l + 16, .. join their sums at the end).  A tile of S^T leaves lane l with
// positions 4 (l / 16) .. + 3, which are the positions the second product takes from that
// lane: the weights go from one product to the next in place, and the value cache keeps
// four positions of a dimension in one word because that word is the other operand.
// Codes go from memory to registers to the matrix cores with no exchange between lanes.
#include "kv8.h"

#include <algorithm>

#include "kv8_plan.h"
#include "launch.h"

namespace wici {

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNoRef = -3e38f;    // ref before the first weight,
constexpr float kNoWeight = -2.99e38f;  // and of rows that see positions, all of weight zero
constexpr float kTopWeight = 6.f;   // log2 of the largest weight when ref is set
constexpr float kMaxWeight = 32768.f;
constexpr float kLeastLog = -68.f;  // below log2 of every scale that is stored
constexpr float kMostScale = 0x1p20f;  // of the values, up to which one reference serves
constexpr float kHugeScore = 16777216.f;
constexpr float kFarBelow = -64.f, kFarStep = 96.f;

// Four codes (bytes b + 128) as fp16 values b: 0x6400 | byte is 1024 + byte, less 1152.
// Both steps are exact.
__device__ __forceinline__ void codes4(unsigned w, unsigned& lo, unsigned& hi) {
  const unsigned p = __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u);
  const unsigned q = __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u);
  const half2_t off = {(_Float16)1152.f, (_Float16)1152.f};
  lo = __builtin_bit_cast(unsigned, __builtin_bit_cast(half2_t, p) - off);
  hi = __builtin_bit_cast(unsigned, __builtin_bit_cast(half2_t, q) - off);
}
__device__ __forceinline__ half8_t codes8(unsigned a, unsigned b) {
  uint4 v;
  codes4(a, v.x, v.y);
  codes4(b, v.z, v.w);
  return __builtin_bit_cast(half8_t, v);
}

// The state of 16 query rows over the positions a wavefront has taken: lane l, row l % 16.
struct RowState {
  float ref = kNoRef, sum = 0.f;  // sum over this lane's positions
  float lift = 0.f;  // the output holds 2^-lift of its sum (whole; 0 while ref serves both)
  bool apart = false;  // the same in all lanes of a row: other rows' values change nothing
};
// Output of 16 rows: tile 4 h + t, element i: dimension 64 h + 16 (l / 16) + 4 i + t.
template <int HD>
using RowOut = floatx4_t[HD / 16];

// Values that are the same in every lane, as scalars: what is read through memory is not
// known to be, and a buffer or a branch that depends on it would run lane by lane.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
template <typename T>
__device__ __forceinline__ T* uniform(T* p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = (uint32_t)uniform((int)(uint32_t)v), hi = (uint32_t)uniform((int)(v >> 32));
  return reinterpret_cast<T*>((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ Kv8Seq uniform(const Kv8Seq& s) {
  return Kv8Seq{uniform(s.base), uniform(s.table), uniform(s.row0), uniform(s.rows), uniform(s.len)};
}

// A thread's index that the compiler does not know to be the same each time around a loop:
// addresses made from it are not kept in registers through the loop.
__device__ __forceinline__ int fresh(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// The codes and scales of a step, as one lane holds them.
template <int HD>
struct Keys {
  uint4 k[kTiles][HD / 64];  // tile t: position l % 16, dimensions (HD / 4) (l / 16) ..
};
template <int HD>
struct Values {
  uint4 v[kTiles][HD / 64];  // positions 4 (l / 16) .. + 3, dimensions 64 h + 4 (l % 16) .. + 3
};
struct Scales {
  float4 k[kTiles], v[kTiles];  // of the keys and values of positions 4 (l / 16) .. + 3
};

// The pages of a step's tiles (-1: none).
struct Pages {
  int phys[kTiles];
  __device__ __forceinline__ bool all() const { return (phys[0] | phys[1]) >= 0; }
};
// A sequence's table entries are read by scalar loads, a chunk or step before they are looked
// at: loads of the vector path would first wait for every row requested before them (2048
// rows of 8192: 344 us, so 313).
__device__ __forceinline__ int entry(const Kv8& c, const Kv8Seq& q, uint32_t pos) {
  typedef const __attribute__((address_space(4))) int32_t* Table;
  return ((Table)(uintptr_t)q.table)[kv8_entry(pos >> c.page_shift, c.max_pages)];
}
// The entries of a step (steps end below 2^31 positions; one past them is still below 2^32).
struct Entries {
  int e[kTiles];
};
__device__ __forceinline__ Entries find(const Kv8& c, const Kv8Seq& q, int step) {
  Entries f;
  f.e[0] = entry(c, q, (uint32_t)step * kStep);
  f.e[1] = c.page_shift >= 5 ? f.e[0] : entry(c, q, (uint32_t)step * kStep + 16);
  return f;
}
__device__ __forceinline__ Pages named(const Kv8& c, const Entries& f) {
  Pages p;
#pragma unroll
  for (int t = 0; t < kTiles; ++t) p.phys[t] = kv8_named(f.e[t], c.n_pages);
  return p;
}

// Addresses are a scalar block base and offset plus a lane's own offset in 32 bits, the same
// for every step.
__device__ __forceinline__ uint4 fetch(__amdgpu_buffer_rsrc_t r, int lane_at, int at) {
  const u32x4_t v = __builtin_amdgcn_raw_buffer_load_b128(r, lane_at, at, 0);
  return make_uint4(v.x, v.y, v.z, v.w);
}
// One KV head of a pool: its key block in page 0, and the bytes from page to page and from a
// key block to its value block.
template <int HD>
struct HeadAt {
  const char* base;
  uint32_t page, values;
  __device__ __forceinline__ HeadAt(const Kv8& c, const Kv8Seq& q, int h)
      : base(q.base + kv8_block_at(0, 0, h, c.n_kv, 1 << c.page_shift, HD)),
        page(2 * c.n_kv * (uint32_t)kv8_block_bytes(1 << c.page_shift, HD)),
        values(page / 2) {}
  __device__ __forceinline__ const char* block(int phys, int which) const {
    return base + (uint64_t)(uint32_t)max(phys, 0) * page + (which ? values : 0);
  }
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const Kv8& c, int phys, int which) const {
    return rsrc(block(phys, which), kv8_block_bytes(1 << c.page_shift, HD));
  }
};
template <int HD>
__device__ __forceinline__ void load_keys(Keys<HD>& s, const Kv8& c, const HeadAt<HD>& at,
                                          const Pages& p, int step, int lane) {
  const int page = 1 << c.page_shift, mine = kv8_key_at(lane & 15, (lane >> 4) * (HD / 4), HD);
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const int slot = (step * kStep + 16 * t) & (page - 1);
    const __amdgpu_buffer_rsrc_t b = at.buffer(c, p.phys[t], 0);
#pragma unroll
    for (int i = 0; i < HD / 64; ++i) s.k[t][i] = fetch(b, mine + 16 * i, kv8_key_at(slot, 0, HD));
  }
}
template <int HD>
__device__ __forceinline__ void load_values(Values<HD>& s, Scales& sl, const Kv8& c,
                                            const HeadAt<HD>& at, const Pages& p, int step,
                                            int lane) {
  const int page = 1 << c.page_shift, g = lane >> 4, mine = kv8_value_at(4 * g, 4 * (lane & 15), HD);
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const int slot = (step * kStep + 16 * t) & (page - 1);
    const __amdgpu_buffer_rsrc_t kb = at.buffer(c, p.phys[t], 0);
    const __amdgpu_buffer_rsrc_t vb = at.buffer(c, p.phys[t], 1);
    sl.k[t] = __builtin_bit_cast(float4, fetch(kb, 16 * g, kv8_scale_at(slot, page, HD)));
    sl.v[t] = __builtin_bit_cast(float4, fetch(vb, 16 * g, kv8_scale_at(slot, page, HD)));
#pragma unroll
    for (int i = 0; i < HD / 64; ++i)
      s.v[t][i] = fetch(vb, mine + 256 * i, kv8_value_at(slot, 0, HD));
  }
}

// S^T of one step: sc[t][i] is the product of position 16 t + 4 (l / 16) + i with row l % 16.
template <int HD, int NT>
__device__ __forceinline__ void scores(floatx4_t (&sc)[kTiles], const Keys<HD>& s,
                                       const half8_t (&qf)[NT][HD / 32]) {
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const unsigned* w = reinterpret_cast<const unsigned*>(&s.k[t][0]);
    sc[t] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) {
      const half8_t a = codes8(w[2 * d], w[2 * d + 1]);
#pragma unroll
      for (int n = 0; n < NT; ++n)
        sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, qf[n][d], sc[t], 0, 0, 0);
    }
  }
}

// The weights of one step from its products (a score is product * key scale * q_unit), as
// NT fp16 terms.  MASKED: some row does not see every position: row l % 16 sees the step's
// positions below `seen`, of the tiles that are there.  `lifts`: some row of the wavefront is
// apart.  Returns whether a row's reference moved: the output so far is then to be multiplied by
// `corr`.  HINT: the compiler is told that moves are rare.  That places the row tiles' code well
// (2048 rows of 8192: 287 us for 304, heads of 64 226 for 236), the split's not (48 tokens at
// 4000, heads of 64, fp32: 45.8 for 44.8).
template <int NT, bool MASKED, bool HINT>
__device__ __forceinline__ bool weights(half8_t (&wf)[NT], RowState& st, bool& lifts,
                                        const floatx4_t (&sc)[kTiles], const Scales& s,
                                        const Pages& p, float q_unit, int seen, int lane,
                                        float& corr) {
  const int left = seen - 4 * (lane >> 4);
  auto on = [&](int t, int i) { return !MASKED || (p.phys[t] >= 0 && 16 * t + i < left); };
  // a score rounded by itself, never joined with what follows: of two that are equal and huge
  // the difference is zero
  auto score = [&](int t, int i) {
    float y = sc[t][i];
    asm volatile("" : "+v"(y));  // (and not for every step, ahead of the rare branches)
    y *= (&s.k[t].x)[i] * q_unit;
    asm volatile("" : "+v"(y));
    return y;
  };
  float sum, most;
  // f(t, i): the exponent of the sum's term; g(t, i, term): the weight (and the term, if another)
  auto weigh = [&](auto f, auto g) {
    sum = most = 0.f;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float e = __builtin_amdgcn_exp2f(on(t, i) ? f(t, i) : -INFINITY);
        float w = on(t, i) ? g(t, i, e) : 0.f;
        // a product rounded once: joined with the conversion below, and not with the
        // difference, the first term is now and then not the one the second completes
        if (NT > 1) asm volatile("" : "+v"(w));
        sum += e;
        most = __builtin_elementwise_maximum(most, w);  // NaN if one is
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const _Float16 term = (_Float16)w;
          wf[n][4 * t + i] = term;
          w -= (float)term;
        }
      }
  };
  auto ahead = [&](int t, int i) {  // a score less the reference
    return __builtin_fmaf(sc[t][i], (&s.k[t].x)[i] * q_unit, -st.ref);
  };
  auto plain = [&]() {
    weigh(ahead, [&](int t, int i, float& e) { return e * (&s.v[t].x)[i]; });
  };
  // The same where some row (`lifts`) has its output's power of two: the weight
  // 2^(y - ref - lift) t, also where 2^(y - ref) alone is below fp32's least: the largest values
  // then outweigh what their softmax weights lack.  Such a term is nothing to the sum.  Rows
  // that are not apart come out as above.
  auto lifted = [&]() {
    bool far = false;
    weigh(
        [&](int t, int i) {
          const float d = st.apart ? score(t, i) - st.ref : ahead(t, i);
          far = st.apart && d < kFarBelow;
          return far ? d + kFarStep : d;
        },
        [&](int t, int i, float& e) {
          const float v = (&s.v[t].x)[i];
          // (one scaling by all the powers of two: no two of them need be within fp32 together)
          const float w = __builtin_amdgcn_ldexpf(
              e * __builtin_amdgcn_frexp_mantf(v),
              __builtin_amdgcn_frexp_expf(v) - (int)st.lift - (far ? (int)kFarStep : 0));
          if (far) e = 0.f;
          __builtin_amdgcn_sched_barrier(0);  // (one after another: registers)
          return w;
        });
  };
  // (rows with lifts move at every step: rare, and one copy less of their code)
  bool move = lifts;
  if (HINT ? __builtin_expect(!move, true) : !move) {
    plain();
    // (NaN: values of scale zero, in memory never appended to, before there is a reference)
    move = __any(!(most <= kMaxWeight));
  }
  if (HINT ? __builtin_expect(move, false) : move) {  // rare after a row's first step
    // the largest of f over this row's positions
    auto largest = [&](auto f) {
      float z = -INFINITY;
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (on(t, i)) z = fmaxf(z, f(t, i));
      z = fmaxf(z, __shfl_xor(z, 16));
      return fmaxf(z, __shfl_xor(z, 32));
    };
    auto lv = [&](int t, int i) {  // (taken here: not for every step, ahead of the branch)
      float x = (&s.v[t].x)[i];
      asm volatile("" : "+v"(x));
      return fmaxf(__builtin_amdgcn_logf(x), kLeastLog);
    };
    const float z = largest([&](int t, int i) { return score(t, i) + lv(t, i); });
    bool large = z != -INFINITY && fabsf(z) > kHugeScore;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) large |= on(t, i) && (&s.v[t].x)[i] > kMostScale;
    const uint64_t lanes = __ballot(large);  // lanes l, l + 16, .. : row l
    const uint32_t two = (uint32_t)lanes | (uint32_t)(lanes >> 32);
    st.apart |= (two | two >> 16) >> (lane & 15) & 1;
    lifts |= __any(st.apart);
    float ref = fmaxf(st.ref, z - kTopWeight), lift = 0.f;
    if (st.apart) {  // (a row's lanes together, so that they still exchange)
      ref = fmaxf(st.ref, largest([&](int t, int i) { return score(t, i); }));
      lift = fmaxf(st.lift + (st.ref - ref),
                   largest([&](int t, int i) { return score(t, i) - ref + lv(t, i); }) - kTopWeight);
      lift = lift > -1e30f ? floorf(lift) : 0.f;  // (0: a row that sees nothing yet)
    }
    st.sum *= __builtin_amdgcn_exp2f(st.ref - ref);
    corr = __builtin_amdgcn_exp2f(st.ref - ref + (st.lift - lift));
    st.ref = ref;
    st.lift = lift;
    if (HINT ? __builtin_expect(lifts, false) : lifts) lifted();
    else plain();
  }
  st.sum += sum;
  return move;
}

// O^T += C^T W^T of one step.
template <int HD, int NT>
__device__ __forceinline__ void add_values(RowOut<HD>& o, const Values<HD>& s,
                                           const half8_t (&wf)[NT]) {
#pragma unroll
  for (int h = 0; h < HD / 64; ++h) {
    const unsigned* v0 = reinterpret_cast<const unsigned*>(&s.v[0][h]);
    const unsigned* v1 = reinterpret_cast<const unsigned*>(&s.v[1][h]);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const half8_t a = codes8(v0[t], v1[t]);
#pragma unroll
      for (int n = 0; n < NT; ++n)
        o[4 * h + t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, wf[n], o[4 * h + t], 0, 0, 0);
    }
  }
}

template <int HD>
__device__ __forceinline__ void rescale(RowOut<HD>& o, float f) {
#pragma unroll
  for (int u = 0; u < HD / 16; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[u][i] *= f;
}

// 16 query rows (row l % 16 of the tile, zero where `on` is false) as NT fp16 terms, each
// row scaled by a power of two that brings its largest finite magnitude into [2^6, 2^7);
// `unit` undoes it.  An element 2^23 below its row's largest is the first that fp16 rounds
// (bf16 rows) or leaves to 2^-31 of that largest.  Infinities and NaN stay in their rows.
template <int HD, int NT>
__device__ __forceinline__ void load_queries(const HeadRows& q, int64_t at, bool on, int lane,
                                             half8_t (&qf)[NT][HD / 32], float& unit) {
  float v[HD / 32][8], most = 0.f;
  at += (lane >> 4) * (HD / 4);
  // (all requested, then all used: one wait)
  if (NT == 1 || q.bf16) {
    uint4 raw[HD / 32];
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
      raw[d] = *reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(q.p) + at + 8 * d);
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t w = (&raw[d].x)[i];
        v[d][2 * i] = __uint_as_float(w << 16);
        v[d][2 * i + 1] = __uint_as_float(w & 0xffff0000u);
      }
  } else {
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float4 x =
            *reinterpret_cast<const float4*>(static_cast<const float*>(q.p) + at + 8 * d + 4 * i);
        v[d][4 * i] = x.x; v[d][4 * i + 1] = x.y; v[d][4 * i + 2] = x.z; v[d][4 * i + 3] = x.w;
      }
  }
#pragma unroll
  for (int d = 0; d < HD / 32; ++d) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[d][i] = on ? v[d][i] : 0.f;
      const float a = fabsf(v[d][i]);
      most = a < INFINITY ? fmaxf(most, a) : most;
    }
  }
  most = fmaxf(most, __shfl_xor(most, 16));
  most = fmaxf(most, __shfl_xor(most, 32));
  const int ex = max((int)(__float_as_uint(most) >> 23) - 127, -120);
  const float up = __uint_as_float((unsigned)(127 + 6 - ex) << 23);
  unit = __uint_as_float((unsigned)(127 - 6 + ex) << 23);
#pragma unroll
  for (int d = 0; d < HD / 32; ++d)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float rest = v[d][i] * up;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        qf[n][d][i] = (_Float16)rest;
        rest -= (float)qf[n][d][i];
      }
    }
}

// A lane's 16 consecutive output values of one half-row.
__device__ __forceinline__ void put_out(const Kv8Attn& a, int row, int head, int d, const float* v) {
  if (!a.out.p) {
    const size_t at = ((size_t)row * a.n_q + head) * a.hd + d;
    store_act4(a.act, at, make_float4(v[0], v[1], v[2], v[3]));
    return;
  }
  const int64_t at = row * a.out.row_stride + head * a.out.head_stride + d;
  if (a.out.bf16) {
    *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.out.p) + at) =
        make_uint2((uint32_t)f32_to_bf16(v[0]) | ((uint32_t)f32_to_bf16(v[1]) << 16),
                   (uint32_t)f32_to_bf16(v[2]) | ((uint32_t)f32_to_bf16(v[3]) << 16));
  } else {
    *reinterpret_cast<float4*>(static_cast<float*>(a.out.p) + at) =
        make_float4(v[0], v[1], v[2], v[3]);
  }
}

// Rows whose weights sum up to nothing though they have positions (`limit` of them, past the
// first that this wavefront takes; `most` the largest limit): where one of those is there, `ref`
// says so.  Rare: their scores are all minus infinity, or their pages absent.  The wavefront
// looks for the sequence's first page together, 64 entries at a time.
__device__ __forceinline__ void note_no_weight(RowState& st, const Kv8& c, const Kv8Seq& q, int limit,
                                               uint32_t past, int most, int lane) {
  const bool none = st.sum == 0.f && (uint32_t)limit > past;
  if (!__any(none)) return;
  const int pages = kv8_steps(most, 1 << c.page_shift);
  for (int p = 0; p < pages; p += 64) {
    const uint64_t there =
        __ballot(p + lane < pages && kv8_page(q.table, p + lane, c.max_pages, c.n_pages) >= 0);
    if (there == 0) continue;
    if (none && (p + __builtin_ctzll(there)) << c.page_shift < limit) st.ref = kNoWeight;
    return;
  }
}

// The joined output of outputs that hold 2^-lift of their sum.
__device__ __forceinline__ void quotient(float (&o)[4], float ref, float lift, float sum) {
  // no position: zeros; only scores of minus infinity: the quotient of two zeros
  const float inv = sum != 0.f ? 1.f / sum : ref == kNoRef ? 0.f : __uint_as_float(0x7fc00000u);
  const float up = __builtin_amdgcn_exp2f(lift);
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = o[i] * inv * up;
}

// Four dimensions of a row of one split: the output where it is the only one, else
// (ref, lift, sum, output) for the merge.  parts: of the launch.
__device__ __forceinline__ void leave(const Kv8Attn& a, int nsplit, int split, size_t parts, int row,
                                      int head, int d, float ref, float lift, float sum,
                                      float (&o)[4]) {
  if (nsplit == 1) {
    quotient(o, ref, lift, sum);
    put_out(a, row, head, d, o);
  } else {
    const size_t at = ((size_t)row * a.n_q + head) * nsplit + split;
    *reinterpret_cast<float4*>(a.work + kv8_part_out(at, a.hd) + d) =
        make_float4(o[0], o[1], o[2], o[3]);
    if (d == 0)
      *reinterpret_cast<float4*>(a.work + kv8_part_state(at, parts, a.hd)) =
          make_float4(ref, lift, sum, 0.f);
  }
}

// ------------------------------------------------------------------- split over positions
// Workgroup (KV head, sequence, split): four wavefronts take the split's steps of 32
// positions in turn for a tile of 16 of the sequence's rows x query heads of the group
// (row r: new row r / G, query head r % G), and are joined at the end.  Splits take
// groups of four steps in turn, so one launch serves any length evenly.  With one
// split the output is written here, otherwise (ref, sum, output) to `part` for the merge.
//
// Bound by the cache's bytes, each read once: 32 tokens at 16384 (40 query on 8 KV heads of
// 128, bf16) 188 us for 1.11 GB, 5.9 TB/s where a large copy moves 5.2; its loads with
// nothing behind them take as long.  Where there is less to read the start, the first loads'
// latency and the join show: 48 tokens at up to 4000 (heads of 64) 36 us for 162 MB, one at
// 16384 (fp32) 14 us for 35 MB.  Three wavefronts a SIMD for heads of 128 (two with two fp16
// terms), four for heads of 64 (with two terms for 12 bytes a lane in scratch: a call of 32 tokens
// at 16384 99 us, with three wavefronts and none 124; 48 at 4000 44 and 43).  256 / 512 / 768 /
// 1024 workgroups: 289 / 203 / 195 / 231 us of the first case, which is why a launch splits no
// further than fills the chip once.
template <int HD, int NT>
__global__ __launch_bounds__(256)
__attribute__((amdgpu_waves_per_eu(HD == 64 ? 4 : NT == 1 ? 3 : 2))) void k_kv8_attn_split(Kv8 c, Kv8Rows r, Kv8Attn a, int nsplit,
                                                        int ntile) {
  __shared__ float s_o[4][16][HD + 4];
  __shared__ float s_ref[4][16], s_lift[4][16], s_sum[4][16];
  const int h = blockIdx.x % c.n_kv, split = blockIdx.x / c.n_kv % nsplit;
  const int tile0 = blockIdx.x / (c.n_kv * nsplit), b = blockIdx.y;
  const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int r16 = lane & 15, G = a.n_q / c.n_kv;
  const Kv8Seq q = uniform(kv8_seq(c, r, b));
  const int64_t cap = (int64_t)c.max_pages << c.page_shift;
  const size_t parts = (size_t)r.n_rows * a.n_q * nsplit;
  // the wavefront's first steps do not depend on the length, so that their pages are
  // looked up beside it
  const HeadAt<HD> kv(c, q, h);
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
    half8_t qf[NT][HD / 32];
    float unit;
    load_queries<HD, NT>(a.q, (q.row0 + rc) * a.q.row_stride + head * a.q.head_stride, on, lane, qf,
                         unit);
    unit *= a.scale * kLog2e;
    RowState st;
    RowOut<HD> o;
    bool lifts = false;
#pragma unroll
    for (int u = 0; u < HD / 16; ++u) o[u] = floatx4_t{0.f, 0.f, 0.f, 0.f};
    if (s < steps) {
      Keys<HD> k;
      Values<HD> v;
      Scales sl;
      Pages now = named(c, e0);
      Entries later = e1;
      load_keys<HD>(k, c, kv, now, s, lane);
      load_values<HD>(v, sl, c, kv, now, s, lane);
      for (;;) {
        floatx4_t sc[kTiles];
        scores<HD, NT>(sc, k, qf);
        const int then = s + stride;
        const Pages next = named(c, later);
        if (then < steps) load_keys<HD>(k, c, kv, next, then, lane);
        half8_t wf[NT];
        float corr = 1.f;
        const bool move =
            s < whole && now.all()
                ? weights<NT, false, false>(wf, st, lifts, sc, sl, now, unit, 0, lane, corr)
                : weights<NT, true, false>(wf, st, lifts, sc, sl, now, unit, limit - s * kStep, lane, corr);
        if (move) rescale<HD>(o, corr);
        add_values<HD, NT>(o, v, wf);
        if (then >= steps) break;
        load_values<HD>(v, sl, c, kv, next, then, lane);
        now = next;
        later = find(c, q, then + stride);
        s = then;
      }
    }
    // join the wavefronts
    st.sum += __shfl_xor(st.sum, 16);
    st.sum += __shfl_xor(st.sum, 32);
    note_no_weight(st, c, q, limit, s0 * kStep, seen(last), lane);
    const int me = fresh(lane), mr = me & 15, mg = me >> 4;
    if (mg == 0) {
      s_ref[wave][mr] = st.ref;
      s_lift[wave][mr] = st.lift;
      s_sum[wave][mr] = st.sum;
    }
#pragma unroll
    for (int hh = 0; hh < HD / 64; ++hh)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(&s_o[wave][mr][64 * hh + 16 * mg + 4 * i]) =
            make_float4(o[4 * hh][i], o[4 * hh + 1][i], o[4 * hh + 2][i], o[4 * hh + 3][i]);
    __syncthreads();
    for (int x = fresh(threadIdx.x); x < 16 * HD / 4; x += 256) {
      const int rr = x / (HD / 4), d = 4 * (x % (HD / 4)), tr = 16 * tile + rr;
      if (tr >= q.rows * G) continue;
      float ref = s_ref[0][rr];
#pragma unroll
      for (int w = 1; w < 4; ++w) ref = fmaxf(ref, s_ref[w][rr]);
      float sum = 0.f, lift = 0.f, all[4] = {};
      bool any = false;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        any |= s_lift[w][rr] != 0.f;
        const float f = __builtin_amdgcn_exp2f(s_ref[w][rr] - ref);
        const float4 v = *reinterpret_cast<const float4*>(&s_o[w][rr][d]);
        sum += f * s_sum[w][rr];
        all[0] += f * v.x; all[1] += f * v.y; all[2] += f * v.z; all[3] += f * v.w;
      }
      if (__builtin_expect(any, false)) {  // the outputs again, each with its power of two
        lift = -INFINITY;
#pragma unroll 1
        for (int w = 0; w < 4; ++w) lift = fmaxf(lift, s_lift[w][rr] + (s_ref[w][rr] - ref));
        lift = floorf(lift);
        all[0] = all[1] = all[2] = all[3] = 0.f;
#pragma unroll 1
        for (int w = 0; w < 4; ++w) {
          const float g = __builtin_amdgcn_exp2f(s_ref[w][rr] - ref + (s_lift[w][rr] - lift));
          const float4 v = *reinterpret_cast<const float4*>(&s_o[w][rr][d]);
          all[0] += g * v.x; all[1] += g * v.y; all[2] += g * v.z; all[3] += g * v.w;
        }
      }
      leave(a, nsplit, split, parts, q.row0 + tr / G, h * G + tr % G, d, ref, lift, sum, all);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------- prompts: row tiles
// Workgroup (KV head, tile of 128 (or 64) rows x query heads, split, sequence): each of
// four wavefronts holds a quarter of the rows and takes every chunk of 64 positions of the
// split.  The codes of a chunk become fp16 operands once for all four, in LDS, lane by lane as
// the products read them (16 bytes a lane, no bank met twice): a wavefront converts a quarter.
// Two buffers: the next chunk's codes are on their way while this one is multiplied, and one
// barrier a chunk parts a buffer's readers from its next writers.
//
// 2048 rows of 8192 positions (32 query on 8 KV heads of 128) take 288 us in bf16, 836 TFLOP/s
// of products where a large fp16 product reaches 1300; 477 us with two fp16 terms.  No unit is
// full: the vector units are busy 52% of the time, the matrix cores 32%, and a wavefront waits
// for operands, products or the other one (the registers allow two a SIMD).  Eight vector
// instructions fewer for 512 scores, and priorities of the products or the weights, changed
// nothing; the next products ahead of the weights need more registers than there are.
template <int HD, int NT, int kRowTiles>
__global__ __launch_bounds__(256)
__attribute__((amdgpu_waves_per_eu(2))) void k_kv8_attn_tile(Kv8 c, Kv8Rows r, Kv8Attn a, int nsplit,
                                                            int ntile) {
  constexpr int DS = HD / 32, DT = HD / 16, kRows = 4 * 16 * kRowTiles;
  static_assert(kRowTiles * NT <= 2, "a step's operands are held in registers");
  __shared__ uint4 s_k[2][kChunkTiles][DS][64];      // keys: tile, 32 dimensions, lane
  __shared__ uint4 s_v[2][kChunkTiles / 2][DT][64];  // values: two tiles, 16 dimensions, lane
  __shared__ float s_scale[2][2][kChunkPos];         // of keys, of values
  const int h = blockIdx.x % c.n_kv, split = blockIdx.x / c.n_kv % nsplit;
  const int tile0 = blockIdx.x / (c.n_kv * nsplit), b = blockIdx.y;
  const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int r16 = lane & 15, g = lane >> 4, G = a.n_q / c.n_kv;
  const Kv8Seq q = uniform(kv8_seq(c, r, b));
  const int64_t cap = (int64_t)c.max_pages << c.page_shift;
  const int page = 1 << c.page_shift;
  const size_t parts = (size_t)r.n_rows * a.n_q * nsplit;
  const int total = q.rows * G, tiles = (total + kRows - 1) / kRows;
  const HeadAt<HD> kv(c, q, h);
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

    RowState st[kRowTiles];
    RowOut<HD> o[kRowTiles];
    bool lifts = false;
#pragma unroll
    for (int x = 0; x < kRowTiles; ++x)
#pragma unroll
      for (int u = 0; u < DT; ++u) o[x][u] = floatx4_t{0.f, 0.f, 0.f, 0.f};

    // what this wavefront brings of a chunk: the keys of tile `wave`; of the pair of tiles
    // wave / 2 the values of half the dimensions (64 dimensions: of half of each word's four);
    // the scales of the keys (wavefront 0) or values (1)
    uint4 kc[HD / 64], vc[2];
    float sc = 0.f;
    int phys[kChunkTiles], later[kChunkTiles];
    const int pair = wave >> 1, half = HD == 128 ? wave & 1 : 0;
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
    auto bring = [&](const int (&p)[kChunkTiles], int chunk) {
      const int j0 = chunk * kChunkPos;
      // p[t], with bits: a choice between the elements would put them into memory
      auto pick = [&](int t) {
        const int lo = p[0] ^ ((p[0] ^ p[1]) & -(t & 1)), hi = p[2] ^ ((p[2] ^ p[3]) & -(t & 1));
        return lo ^ ((lo ^ hi) & -(t >> 1));
      };
      auto keys = [&](__amdgpu_buffer_rsrc_t b, int slot) {
#pragma unroll
        for (int i = 0; i < HD / 64; ++i)
          kc[i] = fetch(b, kv8_key_at(r16, g * (HD / 4), HD) + 16 * i, kv8_key_at(slot, 0, HD));
      };
      auto values = [&](int t, __amdgpu_buffer_rsrc_t b, int slot) {
        vc[t] = fetch(b, kv8_value_at(4 * g, 4 * r16, HD) + 256 * half, kv8_value_at(slot, 0, HD));
      };
      auto scales = [&](const char* block) {
        sc = *(const __attribute__((address_space(1))) float*)(uintptr_t)(
            block + kv8_scale_at((j0 + lane) & (page - 1), page, HD));
      };
      if (whole_chunk) {
        const int slot = j0 & (page - 1);
        keys(kv.buffer(c, p[0], 0), slot + 16 * wave);
        const __amdgpu_buffer_rsrc_t b = kv.buffer(c, p[0], 1);
        values(0, b, slot + 32 * pair);
        values(1, b, slot + 32 * pair + 16);
        if (wave < 2) scales(kv.block(p[0], wave));
      } else {
        keys(kv.buffer(c, pick(wave), 0), (j0 + 16 * wave) & (page - 1));
#pragma unroll
        for (int t = 0; t < 2; ++t)
          values(t, kv.buffer(c, pick(2 * pair + t), 1), (j0 + 32 * pair + 16 * t) & (page - 1));
        if (wave < 2) scales(kv.block(pick(g), wave));
      }
    };
    auto convert = [&](int buf) {
      const unsigned* w = reinterpret_cast<const unsigned*>(kc);
#pragma unroll
      for (int d = 0; d < DS; ++d)
        s_k[buf][wave][d][lane] = __builtin_bit_cast(uint4, codes8(w[2 * d], w[2 * d + 1]));
      const unsigned* v0 = reinterpret_cast<const unsigned*>(&vc[0]);
      const unsigned* v1 = reinterpret_cast<const unsigned*>(&vc[1]);
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (HD == 128 || (t >> 1) == (wave & 1))
          s_v[buf][pair][4 * half + t][lane] = __builtin_bit_cast(uint4, codes8(v0[t], v1[t]));
      if (wave < 2) s_scale[buf][wave][lane] = sc;
    };

    if (c0 < c1) {
      find(c0);
      look();
      bring(phys, c0);
      find(c0 + 1);
    }
    half8_t qf[kRowTiles][NT][DS];
    float unit[kRowTiles];
    int limit[kRowTiles];  // positions each row sees
#pragma unroll
    for (int x = 0; x < kRowTiles; ++x) {
      const int qr = mine + 16 * x + r16, row = qr / G, rc = min(row, q.rows - 1);
      const bool on = qr < total;
      limit[x] = on ? seen(row) : 0;
      load_queries<HD, NT>(a.q, (q.row0 + rc) * a.q.row_stride + (h * G + qr % G) * a.q.head_stride,
                           on, lane, qf[x], unit[x]);
      unit[x] *= a.scale * kLog2e;
    }
    for (int ch = c0; ch < c1; ++ch) {
      const int buf = (ch - c0) & 1;
      int now[kChunkTiles];
#pragma unroll
      for (int t = 0; t < kChunkTiles; ++t) now[t] = phys[t];
      look();
      find(ch + 2);
      convert(buf);
      if (ch + 1 < c1) bring(phys, ch + 1);
      __syncthreads();
      if (ch * kChunkPos >= most) continue;  // past this wavefront's rows
#pragma unroll
      for (int p = 0; p < kChunkTiles / 2; ++p) {
        const int j0 = ch * kChunkPos + 32 * p;
        Pages pg;
        Scales sl;
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
          pg.phys[t] = now[2 * p + t];
          sl.k[t] = *reinterpret_cast<const float4*>(&s_scale[buf][0][32 * p + 16 * t + 4 * g]);
          sl.v[t] = *reinterpret_cast<const float4*>(&s_scale[buf][1][32 * p + 16 * t + 4 * g]);
        }
        // Row tile after row tile: the matrix cores work on one's products while the vector
        // units turn the other's scores into weights.
        floatx4_t x[kRowTiles][kTiles];
        half8_t op[DT];
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
          for (int d = 0; d < DS; ++d)
            op[t * DS + d] = __builtin_bit_cast(half8_t, s_k[buf][2 * p + t][d][lane]);
#pragma unroll
        for (int y = 0; y < kRowTiles; ++y)
#pragma unroll
          for (int t = 0; t < kTiles; ++t) {
            x[y][t] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int d = 0; d < DS; ++d)
#pragma unroll
              for (int n = 0; n < NT; ++n)
                x[y][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(op[t * DS + d], qf[y][n][d],
                                                                 x[y][t], 0, 0, 0);
          }
#pragma unroll
        for (int u = 0; u < DT; ++u) op[u] = __builtin_bit_cast(half8_t, s_v[buf][p][u][lane]);
        const bool whole = least - j0 >= kStep && pg.all();
#pragma unroll
        for (int y = 0; y < kRowTiles; ++y) {
          float corr = 1.f;
          half8_t wf[NT];
          const bool move =
              whole ? weights<NT, false, true>(wf, st[y], lifts, x[y], sl, pg, unit[y], 0, lane, corr)
                    : weights<NT, true, true>(wf, st[y], lifts, x[y], sl, pg, unit[y], limit[y] - j0, lane,
                                        corr);
          if (move) rescale<HD>(o[y], corr);
#pragma unroll
          for (int u = 0; u < DT; ++u)
#pragma unroll
            for (int n = 0; n < NT; ++n)
              o[y][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(op[u], wf[n], o[y][u], 0, 0, 0);
        }
      }
    }
    __syncthreads();  // the buffers are free for the next tile
    const int me = fresh(lane), mg = me >> 4;
#pragma unroll
    for (int y = 0; y < kRowTiles; ++y) {
      st[y].sum += __shfl_xor(st[y].sum, 16);
      st[y].sum += __shfl_xor(st[y].sum, 32);
      note_no_weight(st[y], c, q, limit[y], (uint32_t)c0 * kChunkPos, most, lane);
      const int qr = mine + 16 * y + (me & 15);
      if (qr >= total) continue;
#pragma unroll
      for (int hh = 0; hh < HD / 64; ++hh)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float v[4] = {o[y][4 * hh][i], o[y][4 * hh + 1][i], o[y][4 * hh + 2][i],
                        o[y][4 * hh + 3][i]};
          leave(a, nsplit, split, parts, q.row0 + qr / G, h * G + qr % G,
                64 * hh + 16 * mg + 4 * i, st[y].ref, st[y].lift, st[y].sum, v);
        }
    }
  }
}

// out = sum_s 2^(ref_s + lift_s - ref) o_s / sum_s 2^(ref_s - ref) sum_s over the splits of one
// row and head.  HD / 4 lanes of four dimensions take every P-th split each, P groups of them a
// row and head, and are joined: by a group's lanes alone a head's 128 splits took 43 us one
// after another.
template <int HD>
__global__ __launch_bounds__(256) void k_kv8_attn_merge(Kv8 c, Kv8Rows r, Kv8Attn a, int nsplit) {
  constexpr int L = HD / 4, P = 256 / L;
  __shared__ float4 s_o[P][L];
  __shared__ float4 s_state[P];
  const unsigned u = blockIdx.y * gridDim.x + blockIdx.x;  // (see kv8_merge_grid)
  if (u >= (unsigned)(r.n_rows * a.n_q)) return;
  const int lane = threadIdx.x % L, p = threadIdx.x / L, d = 4 * lane;
  const int row = (int)(u / a.n_q), head = (int)(u % a.n_q);
  if (r.kind == KV8_ARRAYS && r.row_start &&
      (row < r.row_start[0] || row >= r.row_start[r.n_seqs]))
    return;  // a row of no sequence
  const size_t first = (size_t)u * nsplit, parts = (size_t)r.n_rows * a.n_q * nsplit;
  const float4* states = reinterpret_cast<const float4*>(a.work + kv8_part_state(first, parts, HD));
  const float* po = a.work + kv8_part_out(first, HD) + d;
  float ref = kNoRef, lift = 0.f, sum = 0.f, o[4] = {};
  // joins a state and its output to those so far; the lifts where there are any
  bool lifts = false;
  auto join = [&](const float4& m, const float4& v, bool all) {
    const float now = fmaxf(ref, m.x), e = ref - now, g = m.x - now;
    float x = __builtin_amdgcn_exp2f(e), y = __builtin_amdgcn_exp2f(g);
    sum = sum * x + m.z * y;
    if (all) {
      const float up = floorf(fmaxf(lift + e, m.y + g));
      x = __builtin_amdgcn_exp2f(e + (lift - up));
      y = __builtin_amdgcn_exp2f(g + (m.y - up));
      lift = up;
    }
    o[0] = o[0] * x + v.x * y; o[1] = o[1] * x + v.y * y;
    o[2] = o[2] * x + v.z * y; o[3] = o[3] * x + v.w * y;
    ref = now;
    lifts |= m.y != 0.f;
  };
  auto restart = [&]() {
    ref = kNoRef;
    lift = sum = o[0] = o[1] = o[2] = o[3] = 0.f;
  };
#pragma unroll 4
  for (int s = p; s < nsplit; s += P)
    join(states[s], *reinterpret_cast<const float4*>(po + (size_t)s * HD), false);
  if (lifts) {
    restart();
#pragma unroll 1
    for (int s = p; s < nsplit; s += P)
      join(states[s], *reinterpret_cast<const float4*>(po + (size_t)s * HD), true);
  }
  s_o[p][lane] = make_float4(o[0], o[1], o[2], o[3]);
  if (lane == 0) s_state[p] = make_float4(ref, lift, sum, 0.f);
  __syncthreads();
  if (p) return;
  lifts = lift != 0.f;
#pragma unroll
  for (int w = 1; w < P; ++w) join(s_state[w], s_o[w][lane], false);
  if (lifts) {
    restart();
#pragma unroll 1
    for (int w = 0; w < P; ++w) join(s_state[w], s_o[w][lane], true);
  }
  quotient(o, ref, lift, sum);
  put_out(a, row, head, d, o);
}

// ------------------------------------------------------------------- launcher
size_t kv8_attn_floats(int hd, int n_q, int n_kv, int n_seqs, int n_rows, int max_rows,
                       int max_length) {
  const Kv8Plan p = kv8_plan(hd, 1, n_q, n_kv, n_seqs, max_rows, max_length);
  return p.nsplit == 1 ? 0 : kv8_part_floats((size_t)n_rows * n_q * p.nsplit, hd);
}

// (launches that split have at most resident() workgroups of 16 rows x heads, or 2 kCus of 128)
size_t kv8_attn_floats_most(int hd) {
  return kv8_part_floats(std::max(resident(hd, 1) * 16, 2 * kCus * 128), hd);
}

template <int HD>
static hipError_t attn(const Kv8& c, const Kv8Rows& r, const Kv8Attn& a, hipStream_t st, int last) {
  // two fp16 terms unless queries and output are bf16
  const int terms = a.q.bf16 && a.out.p && a.out.bf16 ? 1 : 2;
  const Kv8Plan p = kv8_plan(HD, terms, a.n_q, c.n_kv, r.n_seqs, a.max_rows, a.max_length);
  const int64_t gx = (int64_t)c.n_kv * p.nsplit * p.ntile;
  if (gx > 0x7fffffff || r.n_seqs > 65535 || (p.nsplit > 1 && !a.work)) return hipErrorInvalidValue;
  const dim3 grid((unsigned)gx, r.n_seqs);
  const int edge = p.nsplit == 1 ? last : last & kFirst;
#define WICI_ATTN(...) \
  launch_k((__VA_ARGS__), grid, dim3(256), 0, st, edge, c, r, a, p.nsplit, p.ntile)
  if (p.row_tiles == 2) {
    WICI_ATTN(k_kv8_attn_tile<HD, 1, 2>);
  } else if (p.row_tiles == 1) {
    if (terms == 1) WICI_ATTN(k_kv8_attn_tile<HD, 1, 1>);
    else WICI_ATTN(k_kv8_attn_tile<HD, 2, 1>);
  } else {
    if (terms == 1) WICI_ATTN(k_kv8_attn_split<HD, 1>);
    else WICI_ATTN(k_kv8_attn_split<HD, 2>);
  }
#undef WICI_ATTN
  if (p.nsplit > 1) {
    const int64_t mg = (int64_t)r.n_rows * a.n_q;
    if (mg > 0x7fffffff) return hipErrorInvalidValue;
    const Kv8Merge m = kv8_merge_grid((int)mg);
    launch_k(k_kv8_attn_merge<HD>, dim3(m.x, m.y), dim3(256), 0, st, last & kLast, c, r, a,
             p.nsplit);
  }
  return hipGetLastError();
}

hipError_t launch_kv8_attn(const Kv8& c, const Kv8Rows& r, const Kv8Attn& a, hipStream_t st,
                           int edge) {
  if (a.hd == 128) return attn<128>(c, r, a, st, edge);
  if (a.hd == 64) return attn<64>(c, r, a, st, edge);
  return hipErrorInvalidValue;
}

}  // namespace wici
