// The 4-bit key-value cache as it is written and read back.
//
// 32 neighbouring dimensions share a scale, a power of two: the least with which 7 of it hold
// their largest magnitude.  Division by it is exact, and the conversion instruction rounds the
// quotient to the nearest of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6}, ties to the even code, past 6 to 6
// (checked against the definition for scales over the whole range): codes have one right answer.
#include "kv4.h"
#include "kv_rows.h"

namespace wici {

// The place of a position: its page's block, or nullptr when no page holds it.
template <int HD>
__device__ __forceinline__ char* kv4_block_of(const Kv8& c, const RowAt& w, int which, int h) {
  if (!w.there) return nullptr;
  const int phys = kv8_page(w.table, w.pos >> c.page_shift, c.max_pages, c.n_pages);
  return phys < 0 ? nullptr
                  : w.base + kv4_block_at(phys, which, h, c.n_kv, 1 << c.page_shift, HD);
}

// The largest of a unit's values, by data-parallel moves (a lane and its mirror within 2, 4, 8 and 16).
template <int CTRL>
__device__ __forceinline__ unsigned max_with(unsigned v) {
  return max(v, (unsigned)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, false));
}
template <int LPU>
__device__ __forceinline__ unsigned most_of(unsigned v) {
  v = max_with<kDppHalfMirror>(max_with<kDppXor2>(max_with<kDppXor1>(v)));
  return LPU == 16 ? max_with<kDppMirror>(v) : v;
}

// The codes of a lane's two runs of four dimensions (run a in the low half), and the unit's scale
// bytes, of group g in byte g.  A lane's runs may belong to two groups, and a group to the first
// members of pairs here and the second ones there: every group's maximum is taken over the unit.
template <int LPU>
__device__ __forceinline__ unsigned quantise4(const float (&x)[8], const Runs& run, unsigned& scales) {
  constexpr int NG = LPU / 4;
  const int ga = run.a / kKv4Group, gb = run.b / kKv4Group;
  unsigned ma = 0, mb = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    ma = max(ma, __float_as_uint(x[i]) & 0x7fffffffu);
    mb = max(mb, __float_as_uint(x[4 + i]) & 0x7fffffffu);
  }
  unsigned most = 0, sa = 0, sb = 0;
  scales = 0;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    const unsigned m = most_of<LPU>(max(ga == g ? ma : 0u, gb == g ? mb : 0u));
    const unsigned byte = (unsigned)kv4_scale_byte(m);
    most = max(most, m);
    scales |= byte << (8 * g);
    sa = ga == g ? byte : sa;
    sb = gb == g ? byte : sb;
  }
  // a row holding an infinity or a NaN is kept as NaN, so that what reads it shows it
  if (most >= 0x7f800000u) {
    scales = 0xffffffffu;
    return 0;
  }
  const float fa = __uint_as_float(sa << 23), fb = __uint_as_float(sb << 23);
  unsigned w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], fa, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], fa, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], fb, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], fb, 3);
}

// As the append to the 8-bit cache (and as far from its bytes: 2048 rows of 8 heads of 128, bf16, 8.7
// us for 8.4 MB in and 2.2 out; 48 rows of fp32 with 32 rotated query heads 4.4): a unit takes R neighbouring rows of one head, requested before
// their places are known; four rows of a prompt that are the four positions of a value word write
// it whole.
template <int HD, int R>
__global__ __launch_bounds__(256) void k_kv4_append(Kv8 c, Kv8Rows r, RopeTab rope, int n_q,
                                                    HeadRows q, HeadRows q_out, float q_scale,
                                                    HeadRows k, HeadRows v) {
  constexpr int LPU = HD / 8, UPB = 256 / LPU, NG = HD / kKv4Group;
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
  unsigned code[R], scale[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    blk[i] = kv4_block_of<HD>(c, w[i], is_v, h);
    code[i] = quantise4<LPU>(e[i], run, scale[i]);
  }
  const int slot = w[0].pos & (page - 1);
  const bool word = one_word(w, blk);
  if (is_v && word) {
    unsigned d[4], s = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      d[j] = 0;
#pragma unroll
      for (int i = 0; i < R; ++i) d[j] |= (code[i] >> (8 * j) & 0xffu) << (8 * (i & 3));
    }
    *reinterpret_cast<uint4*>(blk[0] + kv4_value_at(slot, 8 * lane, HD)) =
        make_uint4(d[0], d[1], d[2], d[3]);
    if (lane < NG) {
#pragma unroll
      for (int i = 0; i < R; ++i) s |= (scale[i] >> (8 * lane) & 0xffu) << (8 * (i & 3));
      *reinterpret_cast<unsigned*>(blk[0] + kv4_value_scale_at(slot, lane, page, HD)) = s;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (!blk[i]) continue;
    const int at = w[i].pos & (page - 1);
    if (!is_v) {
      if (run.b == run.a + 4) {
        *reinterpret_cast<unsigned*>(blk[i] + kv4_key_at(at, run.a, HD)) = code[i];
      } else {
        *reinterpret_cast<uint16_t*>(blk[i] + kv4_key_at(at, run.a, HD)) = (uint16_t)code[i];
        *reinterpret_cast<uint16_t*>(blk[i] + kv4_key_at(at, run.b, HD)) = (uint16_t)(code[i] >> 16);
      }
      char* s = blk[i] + kv4_key_scale_at(at, 0, page, HD);
      if (lane == 0) {
        if (NG == 4) *reinterpret_cast<unsigned*>(s) = scale[i];
        else *reinterpret_cast<uint16_t*>(s) = (uint16_t)scale[i];
      }
    } else {
      char* d = blk[i] + kv4_value_at(at, 8 * lane, HD);
#pragma unroll
      for (int j = 0; j < 4; ++j) d[4 * j] = (char)(code[i] >> (8 * j));
      if (lane < NG) blk[i][kv4_value_scale_at(at, lane, page, HD)] = (char)(scale[i] >> (8 * lane));
    }
  }
}

// 2048 rows of 8 heads of 128 to fp32 9.0 us for 2.2 MB in and 16.8 out; 48 rows 3.9.
template <int HD, int R>
__global__ __launch_bounds__(256) void k_kv4_read(Kv8 c, Kv8Rows r, HeadRows k, HeadRows v) {
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
  const int page = 1 << c.page_shift, group = 8 * lane / kKv4Group;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (!w[i].there) continue;
    float e[8] = {};  // a position without a page reads as zero
    if (const char* blk = kv4_block_of<HD>(c, w[i], is_v, h)) {
      const int at = w[i].pos & (page - 1);
      unsigned code, byte;
      if (is_v) {
        const uint4 x = *reinterpret_cast<const uint4*>(blk + kv4_value_at(at & ~3, 8 * lane, HD));
        const int s = 8 * (at & 3);
        code = (x.x >> s & 0xffu) | (x.y >> s & 0xffu) << 8 | (x.z >> s & 0xffu) << 16 |
               (x.w >> s & 0xffu) << 24;
        byte = (unsigned char)blk[kv4_value_scale_at(at, group, page, HD)];
      } else {
        code = *reinterpret_cast<const unsigned*>(blk + kv4_key_at(at, 8 * lane, HD));
        byte = (unsigned char)blk[kv4_key_scale_at(at, group, page, HD)];
      }
      const float scale = __uint_as_float(byte << 23);
#define WICI_PAIR(J)                                                                    \
  {                                                                                     \
    const auto p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, J);            \
    e[2 * J] = p[0];                                                                    \
    e[2 * J + 1] = p[1];                                                                \
  }
      WICI_PAIR(0) WICI_PAIR(1) WICI_PAIR(2) WICI_PAIR(3)
#undef WICI_PAIR
    }
    put44(y, (t + i) * y.row_stride + h * y.head_stride, 8 * lane, 8 * lane + 4, e);
  }
}

// ------------------------------------------------------------------- launchers
hipError_t launch_kv4_append(int hd, const Kv8& c, const Kv8Rows& r, const RopeTab& rope, int n_q,
                             const HeadRows& q, const HeadRows& q_out, float q_scale,
                             const HeadRows& k, const HeadRows& v, hipStream_t st, int edge) {
  if (!q.p) n_q = 0;
  const int R = rows_of_unit(r);
  const unsigned grid = unit_blocks(hd, ((int64_t)r.n_rows + R - 1) / R * (n_q + 2 * c.n_kv));
  if (!grid) return hipErrorInvalidValue;
#define WICI_APPEND(HD, R)                                                                       \
  launch_k(k_kv4_append<HD, R>, dim3(grid), dim3(256), 0, st, edge, c, r, rope, n_q, q, q_out, \
           q_scale, k, v)
  if (hd == 128 && R == 4) WICI_APPEND(128, 4);
  else if (hd == 128) WICI_APPEND(128, 1);
  else if (hd == 64 && R == 4) WICI_APPEND(64, 4);
  else if (hd == 64) WICI_APPEND(64, 1);
  else return hipErrorInvalidValue;
#undef WICI_APPEND
  return hipGetLastError();
}

hipError_t launch_kv4_read(int hd, const Kv8& c, const Kv8Rows& r, const HeadRows& k,
                           const HeadRows& v, hipStream_t st) {
  const int R = rows_of_unit(r);
  const unsigned grid = unit_blocks(hd, ((int64_t)r.n_rows + R - 1) / R * 2 * c.n_kv);
  if (!grid) return hipErrorInvalidValue;
#define WICI_READ(HD, R) \
  launch_k(k_kv4_read<HD, R>, dim3(grid), dim3(256), 0, st, kOnly, c, r, k, v)
  if (hd == 128 && R == 4) WICI_READ(128, 4);
  else if (hd == 128) WICI_READ(128, 1);
  else if (hd == 64 && R == 4) WICI_READ(64, 4);
  else if (hd == 64) WICI_READ(64, 1);
  else return hipErrorInvalidValue;
#undef WICI_READ
  return hipGetLastError();
}

}  // namespace wici
