// Beam search: the k best continuations of each search, and the caches' pages put in their order.
//
// A continuation of beam i (score c_i, logits z_i) by word v has the score
//   s_iv = c_i + ((z_iv - m_i) - L_i),   m_i = max_u z_iu,   L_i = log sum_u e^(z_iu - m_i),
// and of all (i, v) of a search the k greatest are chosen, equal ones by the lowest (i, v).  (In this
// order beams whose logits are alike up to a constant have equal scores, not nearly equal ones.)
//
// Within a beam the order is that of the logits and needs no L_i; between beams it does, and two
// continuations may be as near each other as numbers of 24 bits get: L_i and s_iv are formed in 64
// bits, and from parts of a row that its length alone decides, so that beams that are alike have the
// same ones.  64-bit multiply-adds run at the rate of 32-bit ones here.
//
// One pass over the logits (k_beam_scan) leaves, for each unit of 2 KiB, its largest logit and the
// sum of exponentials against it, and for each group of 64 x 16 bytes (more of a vocabulary past
// 2^18 fp32 logits) its largest logit.  The k first elements of a row are in the k groups with the
// largest maxima (of equal maxima the first groups): any other group has k elements before its
// own.  So k_beam_rows sorts the groups' maxima, reads the k groups again, and sorts what of them
// is not below the k-th maximum; k_beam_join puts the beams' first k together.
#include "beam.h"

#include "beam_plan.h"
#include "launch.h"

namespace wici {

// ------------------------------------------------------------------- elements
// A row as blocks of E elements, counted from its first one wherever that lies: rows that are alike
// are cut alike, and have the same sums to the last bit.  (Loads of 16 bytes take any alignment.)
template <bool BF16>
struct Logits {
  static constexpr int E = BF16 ? 8 : 4;  // of a block of 16 bytes
  const char* base;
  int vocab;
  int to;  // the blocks that the row has whole: 0 .. to - 1
  __device__ __forceinline__ Logits(const void* p, int64_t row_stride, int row, int vocab_)
      : base(static_cast<const char*>(p) + row * row_stride * (BF16 ? 2 : 4)), vocab(vocab_),
        to(vocab_ / E) {}
  __device__ __forceinline__ int index(int b) const { return b * E; }  // of its first element
  __device__ __forceinline__ uint4 whole(int b) const {
    uint4 w;
    __builtin_memcpy(&w, base + 16 * (int64_t)b, 16);
    return w;
  }
  __device__ __forceinline__ void unpack(const uint4& w, float (&z)[E]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x = (&w.x)[i];
      if constexpr (BF16) {
        z[2 * i] = __uint_as_float(x << 16);
        z[2 * i + 1] = __uint_as_float(x & 0xffff0000u);
      } else {
        z[i] = __uint_as_float(x);
      }
    }
  }
  // The block that the row ends in, element by element; -inf where it has none.
  __device__ __forceinline__ void part(int b, float (&z)[E]) const {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      z[i] = -INFINITY;
      if (index(b) + i < vocab) {
        if constexpr (BF16) z[i] = bf16_to_f32(reinterpret_cast<const bf16_t*>(base)[index(b) + i]);
        else z[i] = reinterpret_cast<const float*>(base)[index(b) + i];
      }
    }
  }
  // N blocks, `step` apart from b on: those that are whole requested together.
  template <int N>
  __device__ __forceinline__ void blocks(int b, int step, float (&z)[N][E]) const {
    uint4 w[N];
    const bool any = to > 0;  // (the same in every lane)
#pragma unroll
    for (int n = 0; n < N; ++n) w[n] = any ? whole(min(b + n * step, to - 1)) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int n = 0; n < N; ++n) unpack(w[n], z[n]);
    if (__all(b + (N - 1) * step < to)) return;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int at = b + n * step;
      if (at >= to)
#pragma unroll
        for (int i = 0; i < E; ++i) z[n][i] = -INFINITY;
      if (at == to) part(at, z[n]);
    }
  }
};

// e^x for x <= 0 to 2^-52 + |x| 2^-54 of itself, and 1 for 0 (what is below e^-200 counts as that): x =
// n ln 2 + r with |r| <= ln 2 / 2, and 1 + r + r^2 p(r) with the polynomial p of degree 9 that meets
// (e^r - 1 - r) / r^2 at the ten Chebyshev nodes of that range (2^-55).  Added to 1.5 2^52, n stands in
// the sum's low bits; it goes into the exponent, which stays in its range.  (A degree of 7, errors of 2^-34,
// took 19.7 us for 23.0 below and reached the scores: those of all but certain words were 1e-10 off.)
__device__ __forceinline__ double exp_below(double x) {
  x = fmax(x, -200.0);
  const double t = __builtin_fma(x, 1.4426950408889634074, 0x1.8p52);
  const double r = __builtin_fma(t - 0x1.8p52, -0.69314718055994530942, x);
  double p = 2.5100375832561234e-08;
  p = __builtin_fma(p, r, 2.7620075879983367e-07);
  p = __builtin_fma(p, r, 2.7557268480310024e-06);
  p = __builtin_fma(p, r, 2.4801521322368692e-05);
  p = __builtin_fma(p, r, 0.00019841269863040545);
  p = __builtin_fma(p, r, 0.0013888888917196719);
  p = __builtin_fma(p, r, 0.008333333333330065);
  p = __builtin_fma(p, r, 0.041666666666624164);
  p = __builtin_fma(p, r, 0.16666666666666669);
  p = __builtin_fma(p, r, 0.5000000000000001);
  p = __builtin_fma(p, r, 1.0);
  p = __builtin_fma(p, r, 1.0);
  return __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, p) + (__builtin_bit_cast(uint64_t, t) << 52));
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m);
  return v;
}

// ------------------------------------------------------------------- the pass over the logits
// A wavefront takes a unit, kLoads blocks a lane at a time.  A NaN or an infinity makes the sum NaN.
//
// Bound by the exponentials: 19 instructions an element, vector units busy 85% of the time.  128 rows of
// 152064 bf16 logits 23.0 us for 39 MB (the instructions alone 15, the bytes 7.5), 4 of 128256 in fp32 3.9.
template <bool BF16>
__global__ __launch_bounds__(256) void k_beam_scan(BeamSelect a, BeamPlan p, double* __restrict__ sums,
                                                   float* __restrict__ tops,
                                                   float* __restrict__ groups) {
  constexpr int E = Logits<BF16>::E;
  const int row = blockIdx.y, lane = threadIdx.x & 63;
  const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (unit >= p.units) return;
  const Logits<BF16> z(a.logits, a.row_stride, row, a.vocab);
  float top = -INFINITY, group = -INFINITY;
  double sum = 0.0;  // of this lane, against `top`
  bool bad = false;
  for (int l0 = 0; l0 < p.per_unit; l0 += kLoads) {
    const int first = unit * p.per_unit + l0;
    float x[kLoads][E];
    z.template blocks<kLoads>(first * 64 + lane, 64, x);
    float most[kLoads], now = top;
#pragma unroll
    for (int l = 0; l < kLoads; ++l) {
      most[l] = x[l][0];
#pragma unroll
      for (int i = 1; i < E; ++i) most[l] = __builtin_elementwise_maximum(most[l], x[l][i]);
      bad |= !(most[l] < INFINITY);  // (NaN if one is)
      most[l] = wave_max(most[l]);
      now = fmaxf(now, most[l]);
      group = fmaxf(group, most[l]);
      const int load = first + l + 1;
      if ((load & (p.per_group - 1)) == 0) {  // the group's last
        const int g = load / p.per_group - 1;
        if (lane == 0 && g < p.groups) groups[(size_t)row * p.groups + g] = group;
        group = -INFINITY;
      }
    }
    if (now == -INFINITY) continue;  // nothing yet
    sum *= exp_below((double)top - (double)now);  // (from -inf: of nothing)
    top = now;
#pragma unroll
    for (int l = 0; l < kLoads; ++l)
#pragma unroll
      for (int i = 0; i < E; ++i) sum += exp_below((double)x[l][i] - (double)top);
  }
  sum = wave_sum64(sum);
  if (__any(bad)) sum = __builtin_nan("");
  if (lane == 0) {
    const size_t at = (size_t)row * p.units + unit;
    tops[at] = top;
    sums[at] = sum;
  }
}

// ------------------------------------------------------------------- sorted lists
// A key orders by value, then by the lowest index; 0 is none.
__device__ __forceinline__ uint64_t key_of(float z, uint32_t index) {
  const uint32_t b = __float_as_uint(z + 0.f);  // (-0 and 0 are equal)
  const uint32_t o = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
  return (uint64_t)o << 32 | (0xffffffffu - index);
}
__device__ __forceinline__ float value_of(uint64_t key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float(o ^ (o >> 31 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ uint32_t index_of(uint64_t key) { return 0xffffffffu - (uint32_t)key; }

// The key of lane l ^ M.  Within 16 lanes by data-parallel moves of the vector unit, past them by its
// exchange of rows: the LDS crossbar would cost several times as much a step.
template <int CTRL, int BANKS>
__device__ __forceinline__ uint32_t move_lanes(uint32_t old, uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)v, CTRL, 0xf, BANKS, false);
}
template <int M>
__device__ __forceinline__ uint32_t other_lane(uint32_t v) {
  if constexpr (M == 1) return move_lanes<kDppXor1, 0xf>(v, v);
  else if constexpr (M == 2) return move_lanes<kDppXor2, 0xf>(v, v);
  else if constexpr (M == 4)  // four lanes on (banks 0 and 2) or back (1 and 3)
    return move_lanes<0x114, 0xa>(move_lanes<0x104, 0x5>(v, v), v);
  else if constexpr (M == 8) return move_lanes<0x128, 0xf>(v, v);  // eight around the row
  else if constexpr (M == 16) {
    const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return threadIdx.x & 16 ? p[0] : p[1];
  } else {
    const auto p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return threadIdx.x & 32 ? p[0] : p[1];
  }
}
template <int M>
__device__ __forceinline__ uint64_t other_lane(uint64_t v) {
  return (uint64_t)other_lane<M>((uint32_t)(v >> 32)) << 32 | other_lane<M>((uint32_t)v);
}
// Steps of a bitonic network over the 64 lanes: of lanes l and l ^ M the one with bit M clear keeps
// the larger key where the run of RUN lanes falls (64: everywhere).
template <int RUN, int M>
__device__ __forceinline__ uint64_t steps64(uint64_t v, int lane) {
  const uint64_t w = other_lane<M>(v);
  const bool larger = ((lane & M) == 0) == (RUN == 64 || (lane & RUN) == 0);
  v = (v > w) == larger ? v : w;
  if constexpr (M > 1) return steps64<RUN, M / 2>(v, lane);
  else return v;
}
// The lanes' keys in falling order.
__device__ __forceinline__ uint64_t sort64(uint64_t v, int lane) {
  v = steps64<2, 1>(v, lane);
  v = steps64<4, 2>(v, lane);
  v = steps64<8, 4>(v, lane);
  v = steps64<16, 8>(v, lane);
  v = steps64<32, 16>(v, lane);
  return steps64<64, 32>(v, lane);
}
// The first 64 of two falling lists, in falling order; w: the other list's key of lane 63 - l.
__device__ __forceinline__ uint64_t merge64(uint64_t v, uint64_t w, int lane) {
  return steps64<64, 32>(v > w ? v : w, lane);
}
// The first 64 of the lists of `waves` wavefronts, to the first one.
template <int WAVES>
__device__ __forceinline__ uint64_t merge_waves(uint64_t v, uint64_t (*list)[64], int wave, int lane) {
  list[wave][lane] = v;
#pragma unroll
  for (int step = 1; step < WAVES; step *= 2) {
    __syncthreads();
    if (wave % (2 * step) == 0) {
      v = merge64(v, list[wave + step][63 - lane], lane);
      list[wave][lane] = v;
    }
  }
  __syncthreads();
  return v;
}

// Between a wavefront's writes to its part of LDS and its reads of them by other lanes.
__device__ __forceinline__ void own_writes() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ------------------------------------------------------------------- a beam's first k
// One workgroup a row: m_i and L_i, and the row's first k logits with their words.  Bound by latencies,
// one after another: the maxima's load, two sorts and trees of merges, the groups' loads: 10.3 us for
// 128 rows, 9.7 for 4 (12 where the networks exchanged keys through the LDS crossbar).
constexpr int kRowWaves = kMostGroups / 64;
template <bool BF16>
__global__ __launch_bounds__(64 * kRowWaves) void k_beam_rows(BeamSelect a, BeamPlan p,
                                                            const double* __restrict__ sums,
                                                            const float* __restrict__ tops,
                                                            const float* __restrict__ groups,
                                                            double* __restrict__ lse,
                                                            float* __restrict__ row_top,
                                                            float* __restrict__ out_z,
                                                            int32_t* __restrict__ out_index) {
  constexpr int E = Logits<BF16>::E;
  __shared__ uint64_t s_list[kRowWaves][64];
  __shared__ uint64_t s_hold[kRowWaves][128];
  __shared__ float s_top[kRowWaves];
  __shared__ double s_sum[kRowWaves];
  const int row = blockIdx.x, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = threadIdx.x;

  // the groups in the order of their maxima
  uint64_t v = t < p.groups ? key_of(groups[(size_t)row * p.groups + t], t) : 0;
  // (p.units is at most as many as groups)
  const float top = t < p.units ? tops[(size_t)row * p.units + t] : -INFINITY;
  const double sum = t < p.units ? sums[(size_t)row * p.units + t] : 0.0;
  const float wtop = wave_max(top);
  if (lane == 0) s_top[wave] = wtop;
  v = merge_waves<kRowWaves>(sort64(v, lane), s_list, wave, lane);
  // (s_list[0] holds the first 64 groups; its barriers stand between s_top's writes and reads)
  float most = s_top[0];
#pragma unroll
  for (int w = 1; w < kRowWaves; ++w) most = fmaxf(most, s_top[w]);
  // a unit of nothing has sum 0; NaN sums stay
  const double part = wave_sum64(top == -INFINITY ? sum : sum * exp_below((double)top - (double)most));
  if (lane == 0) s_sum[wave] = part;

  // of the first k groups, what is not below the k-th maximum
  const uint64_t last = s_list[0][a.k - 1];
  const uint32_t least = (uint32_t)(last >> 32);
  const int n_groups = min(a.k, p.groups);
  const Logits<BF16> z(a.logits, a.row_stride, row, a.vocab);
  uint64_t best = 0;
  int held = 0;
  uint64_t* hold = s_hold[wave];
  // (falling lists both: one of them turned around)
  auto take = [&](uint64_t k) {
    hold[lane] = sort64(k, lane);
    own_writes();
    best = merge64(best, hold[63 - lane], lane);
  };
  for (int g = wave; g < n_groups; g += kRowWaves) {
    const int group = (int)index_of(s_list[0][g]);
    for (int l = 0; l < p.per_group; ++l) {
      float x[1][E];
      const int b = (group * p.per_group + l) * 64 + lane, at = z.index(b);
      z.template blocks<1>(b, 0, x);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        // (a block's places outside the row are -inf, as masked words are: neither is a candidate)
        const uint64_t key = key_of(x[0][i], (uint32_t)(at + i));
        const bool on = x[0][i] != -INFINITY && (uint32_t)(key >> 32) >= least;
        const uint64_t lanes = __ballot(on);
        if (!lanes) continue;
        if (on) hold[held + __popcll(lanes & ((1ull << lane) - 1))] = key;
        held += __popcll(lanes);
        if (held >= 64) {
          own_writes();
          take(hold[lane]);
          held -= 64;
          const uint64_t rest = hold[64 + lane];
          own_writes();
          hold[lane] = rest;
        }
      }
    }
  }
  own_writes();
  if (held) take(lane < held ? hold[lane] : 0);
  __syncthreads();  // s_list is read no more
  if (t == 64 * kRowWaves - 1) {  // (of a wavefront that the merge needs only once)
    double all = s_sum[0];
#pragma unroll
    for (int w = 1; w < kRowWaves; ++w) all += s_sum[w];
    lse[row] = most == -INFINITY && all == 0.0 ? 0.0 : log(all);
    row_top[row] = most;
  }
  best = merge_waves<kRowWaves>(best, s_list, wave, lane);
  if (wave) return;
  if (lane < a.k) {
    const size_t at = (size_t)row * a.k + lane;
    out_z[at] = best ? value_of(best) : -INFINITY;
    out_index[at] = best ? (int)index_of(best) : -1;
  }
}

// ------------------------------------------------------------------- a search's first k
// Of the beams' lists, each in falling order: a candidate's place is the number before it in its
// own list and, by bisection, in each other: a work-item finds one of those numbers.  Equal scores: the
// lower beam first.  (16 searches of 8 beams, k 16: 4.0 us; each candidate's numbers one after another
// 6.9.)
constexpr int kJoin = 1024;
__global__ __launch_bounds__(kJoin) void k_beam_join(BeamSelect a, const double* __restrict__ lse,
                                                     const float* __restrict__ row_top,
                                                     const float* __restrict__ z,
                                                     const int32_t* __restrict__ index) {
  __shared__ double s_score[kMostBeams * kMostChosen];
  __shared__ int s_place[kMostBeams * kMostChosen];
  __shared__ int s_count[kMostBeams];  // live candidates of a beam: the first ones of its list
  __shared__ int s_bad, s_all;
  const int b = blockIdx.x, W = a.beams, k = a.k, t = threadIdx.x;
  if (t < W) s_count[t] = 0;
  if (t == 0) s_bad = s_all = 0;
  __syncthreads();
  for (int x = t; x < W * k; x += kJoin) {
    const int i = x / k, r = x % k;
    const size_t row = (size_t)b * W + i;
    const float c = a.scores[row], zz = z[row * k + r], top = row_top[row];
    const double l = lse[row];
    const bool live = c != -INFINITY;
    // (a beam that is not alive may hold anything)
    if (live && (!(c < INFINITY) || l != l)) s_bad = 1;
    const bool on = live && zz != -INFINITY;
    s_score[x] = on ? (double)c + (((double)zz - (double)top) - l) : -INFINITY;
    s_place[x] = r;
    if (on) {
      atomicAdd(&s_count[i], 1);
      atomicAdd(&s_all, 1);
    }
  }
  __syncthreads();
  const bool bad = s_bad != 0;
  const size_t to = (size_t)b * k;
  if (t < k && (bad || t >= s_all)) {
    a.out_scores[to + t] = bad ? __uint_as_float(0x7fc00000u) : -INFINITY;
    a.out_parent[to + t] = a.out_token[to + t] = -1;
  }
  if (bad) return;
  for (int y = t; y < W * k * W; y += kJoin) {
    const int j = y / (W * k), x = y % (W * k), i = x / k;
    if (i == j || x % k >= s_count[i]) continue;
    const double s = s_score[x];
    int lo = 0, hi = s_count[j];  // candidates before lo are before this one, from hi on not
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      const double m = s_score[j * k + mid];
      if (m > s || (m == s && j < i)) lo = mid + 1;
      else hi = mid;
    }
    atomicAdd(&s_place[x], lo);
  }
  __syncthreads();
  for (int x = t; x < W * k; x += kJoin) {
    const int i = x / k, r = x % k, place = s_place[x];
    if (r >= s_count[i] || place >= k) continue;
    a.out_scores[to + place] = (float)s_score[x];
    a.out_parent[to + place] = i;
    a.out_token[to + place] = index[((size_t)b * W + i) * k + r];
  }
}

hipError_t launch_beam_select(const BeamSelect& a, hipStream_t st) {
  const BeamPlan p = beam_plan(a.vocab, a.bf16);
  const int64_t rows = (int64_t)a.n * a.beams;
  if (rows < 1 || rows > kMostRows || a.k < 1 || a.k > kMostChosen || a.beams > kMostBeams ||
      p.groups > kMostGroups || p.units > kMostGroups || !a.work)
    return hipErrorInvalidValue;
  const BeamSpace s = beam_space(p, rows, a.k);
  double* sums = reinterpret_cast<double*>(a.work + s.sum);
  double* lse = reinterpret_cast<double*>(a.work + s.lse);
  float* tops = reinterpret_cast<float*>(a.work + s.top);
  float* groups = reinterpret_cast<float*>(a.work + s.group);
  float* row_top = reinterpret_cast<float*>(a.work + s.row_top);
  float* z = reinterpret_cast<float*>(a.work + s.z);
  int32_t* index = reinterpret_cast<int32_t*>(a.work + s.index);
  const dim3 scan((p.units + 3) / 4, (unsigned)rows);
#define WICI_BEAM(B)                                                                            \
  launch_k(k_beam_scan<B>, scan, dim3(256), 0, st, kFirst, a, p, sums, tops, groups);           \
  launch_k(k_beam_rows<B>, dim3((unsigned)rows), dim3(64 * kRowWaves), 0, st, 0, a, p, sums, tops, \
           groups, lse, row_top, z, index)
  if (a.bf16) {
    WICI_BEAM(true);
  } else {
    WICI_BEAM(false);
  }
#undef WICI_BEAM
  launch_k(k_beam_join, dim3(a.n), dim3(kJoin), 0, st, kLast, a, lse, row_top,
           z, index);
  return hipGetLastError();
}

// ------------------------------------------------------------------- reordering
// Beam i of a search continues the one that was `parent`: it shares that one's whole pages through
// the table, and the last, partial one, which each beam writes on by itself, is copied into the
// beam's spare page.  Pages that are written (spares) are no beam's, so copies wait for nothing;
// the tables change in a second launch, after all copies have read them.
struct BeamMove {
  bool on;
  int src;         // the parent's sequence
  int full, tail;  // whole pages, positions of the partial one
};
__device__ __forceinline__ BeamMove beam_move(const Kv8& c, int seq, int beams,
                                              const int32_t* __restrict__ parent,
                                              const int32_t* __restrict__ length) {
  const int first = seq / beams * beams, p = parent[seq];
  const int64_t cap = (int64_t)c.max_pages << c.page_shift;
  const int n = (int)min((int64_t)max(length[first], 0), cap);
  return BeamMove{p >= 0 && p < beams && first + p != seq, first + p, n >> c.page_shift,
                  n & ((1 << c.page_shift) - 1)};
}

struct BeamPools {
  char* pool[kPoolsALaunch];
};
// A work-item copies 16 bytes, past the caches: nothing here is read again soon.  (Four a work-item, 4 KiB
// apart and through the caches, took 20.3 us for 8.5 over the caches of 32 layers, 13.4 MB in all.)
__global__ __launch_bounds__(256) void k_beam_copy(Kv8 c, BeamPools pools, size_t page_bytes, int beams,
                                                   const int32_t* __restrict__ parent,
                                                   const int32_t* __restrict__ length,
                                                   const int32_t* __restrict__ spare) {
  const int seq = blockIdx.y;
  const BeamMove m = beam_move(c, seq, beams, parent, length);
  if (!m.on || !m.tail) return;
  const int from = kv8_page(c.table + m.src * c.table_stride, m.full, c.max_pages, c.n_pages);
  const int to = kv8_named(spare[seq], c.n_pages);
  if (from < 0 || to < 0 || from == to) return;
  char* pool = pools.pool[blockIdx.z];
  const u32x4_t* x = reinterpret_cast<const u32x4_t*>(pool + (size_t)from * page_bytes);
  u32x4_t* y = reinterpret_cast<u32x4_t*>(pool + (size_t)to * page_bytes);
  const size_t at = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (at < page_bytes / 16) __builtin_nontemporal_store(__builtin_nontemporal_load(x + at), y + at);
}

// A work-item takes one entry of all tables of a search: reads every beam's, then writes.
constexpr int kEntries = 128;
__global__ __launch_bounds__(kEntries) void k_beam_tables(Kv8 c, int beams,
                                                          const int32_t* __restrict__ parent,
                                                          const int32_t* __restrict__ length,
                                                          int32_t* __restrict__ table,
                                                          int32_t* __restrict__ spare) {
  __shared__ int32_t s_old[kMostBeams][kEntries];
  const int t = threadIdx.x, first = blockIdx.y * beams;
  const int64_t j = (int64_t)blockIdx.x * kEntries + t;
  const BeamMove m = beam_move(c, first, beams, parent, length);
  if (j > m.full || j >= c.max_pages || (j == m.full && !m.tail)) return;
  for (int i = 0; i < beams; ++i) s_old[i][t] = table[(first + i) * c.table_stride + j];
  for (int i = 0; i < beams; ++i) {
    const int p = parent[first + i];
    if (p < 0 || p >= beams || p == i) continue;
    int32_t now = s_old[p][t];
    if (j == m.full && kv8_named(now, c.n_pages) >= 0) {
      now = spare[first + i];
      spare[first + i] = s_old[i][t];
    }
    table[(first + i) * c.table_stride + j] = now;
  }
}

hipError_t launch_beam_reorder(const Kv8& c, size_t page_bytes, void* const* pools, int n_pools,
                               int n, int beams, const int32_t* parent, const int32_t* length,
                               int32_t* table, int32_t* spare, hipStream_t st) {
  const int64_t seqs = (int64_t)n * beams;
  if (seqs < 1 || seqs > 65535 || beams > kMostBeams || page_bytes % 16) return hipErrorInvalidValue;
  const size_t gx = (page_bytes / 16 + 255) / 256;
  if (gx > 0x7fffff) return hipErrorInvalidValue;
  for (int at = 0; at < n_pools; at += kPoolsALaunch) {
    BeamPools p{};
    const int here = n_pools - at < kPoolsALaunch ? n_pools - at : kPoolsALaunch;
    for (int i = 0; i < here; ++i) p.pool[i] = static_cast<char*>(pools[at + i]);
    launch_k(k_beam_copy, dim3((unsigned)gx, (unsigned)seqs, here), dim3(256), 0, st,
             at == 0 ? kFirst : 0, c, p, page_bytes, beams, parent, length, spare);
  }
  launch_k(k_beam_tables, dim3((unsigned)((c.max_pages + kEntries - 1) / kEntries), n),
           dim3(kEntries), 0, st, n_pools ? kLast : kOnly, c, beams, parent, length, table, spare);
  return hipGetLastError();
}

}  // namespace wici
