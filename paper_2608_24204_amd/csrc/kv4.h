// The 4-bit key-value cache and the operators around it, as the host code and the kernels see
// them.  A cache, its rows and its attention are described as the 8-bit one's.
#pragma once
#include <hip/hip_runtime.h>

#include "kv4_layout.h"
#include "kv8.h"

namespace wici {

hipError_t launch_kv4_append(int hd, const Kv8& c, const Kv8Rows& r, const RopeTab& rope, int n_q,
                             const HeadRows& q, const HeadRows& q_out, float q_scale,
                             const HeadRows& k, const HeadRows& v, hipStream_t st,
                             int edge = 3);
hipError_t launch_kv4_read(int hd, const Kv8& c, const Kv8Rows& r, const HeadRows& k,
                           const HeadRows& v, hipStream_t st);
size_t kv4_attn_floats(int hd, int n_q, int n_kv, int n_seqs, int n_rows, int max_rows,
                       int max_length);
hipError_t launch_kv4_attn(const Kv8& c, const Kv8Rows& r, const Kv8Attn& a, hipStream_t st,
                           int edge = 3);

}  // namespace wici
