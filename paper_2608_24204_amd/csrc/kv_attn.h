// What the attention kernels over the paged caches share: scalar page look-ups, where a wavefront's
// results go, and the join of a row's partial results.
#pragma once
#include "kv8.h"
#include "kv8_plan.h"

namespace wici {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNoRef = -3e38f;    // ref before the first weight,
constexpr float kNoWeight = -2.99e38f;  // and of rows that see positions, all of weight zero

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
__device__ __forceinline__ void note_no_weight(float& ref, float sum, const Kv8& c, const Kv8Seq& q,
                                               int limit, uint32_t past, int most, int lane) {
  const bool none = sum == 0.f && (uint32_t)limit > past;
  if (!__any(none)) return;
  const int pages = kv8_steps(most, 1 << c.page_shift);
  for (int p = 0; p < pages; p += 64) {
    const uint64_t there =
        __ballot(p + lane < pages && kv8_page(q.table, p + lane, c.max_pages, c.n_pages) >= 0);
    if (there == 0) continue;
    if (none && (p + __builtin_ctzll(there)) << c.page_shift < limit) ref = kNoWeight;
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

// out = sum_s 2^(ref_s + lift_s - ref) o_s / sum_s 2^(ref_s - ref) sum_s: the merge of a launch that
// split its positions (kv8_attn.hip).
hipError_t launch_kv_attn_merge(int hd, const Kv8& c, const Kv8Rows& r, const Kv8Attn& a, int nsplit,
                                hipStream_t st, int edge);

}  // namespace wici
