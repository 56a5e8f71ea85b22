// C entry points of the operators on caller-owned tensors: argument checks, then one
// launcher call.  Nothing here allocates or waits, and nothing throws.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/wici.h"
#include "kv8.h"
#include "rope.h"

namespace {

using wici::HeadRows;
using wici::Kv8;
using wici::Kv8Rows;
using wici::RopeTab;

// Makes the stream's GPU current for the call (the null stream belongs to whichever
// already is).
class OnDeviceOf {
 public:
  explicit OnDeviceOf(void* stream) {
    if (!stream) return;
    hipDevice_t dev = 0;
    int cur = 0;
    err_ = hipStreamGetDevice(static_cast<hipStream_t>(stream), &dev);
    if (err_ == hipSuccess) err_ = hipGetDevice(&cur);
    if (err_ != hipSuccess || cur == dev) return;
    err_ = hipSetDevice(dev);
    if (err_ == hipSuccess) back_ = cur;
  }
  ~OnDeviceOf() {
    if (back_ >= 0) (void)hipSetDevice(back_);
  }
  OnDeviceOf(const OnDeviceOf&) = delete;
  bool ok() const { return err_ == hipSuccess; }

 private:
  hipError_t err_ = hipSuccess;
  int back_ = -1;
};

// Head rows a grid of one launch takes: 16 threads each, 2^32 in all; and of the attention,
// whose partial results are joined by a workgroup a row and head.
constexpr int64_t kMostAttended = 1 << 24;
bool units_ok(int64_t rows, int64_t heads) { return rows * heads < (int64_t)1 << 28; }

bool aligned(const void* p) { return p && (uintptr_t)p % 16 == 0; }

bool rows_ok(const wici_head_rows& x, int64_t heads, int64_t head_dim) {
  return aligned(x.data) && (x.dtype == WICI_F32 || x.dtype == WICI_BF16) &&
         x.row_stride > 0 && x.head_stride > 0 && x.row_stride % 8 == 0 &&
         x.head_stride % 8 == 0 && x.row_stride <= (int64_t)1 << 40 &&
         x.head_stride <= (int64_t)1 << 40 &&
         (heads == 1 || x.head_stride >= head_dim) && x.row_stride >= head_dim;
}
HeadRows rows_of(const wici_head_rows& x) {
  return HeadRows{x.data, x.dtype == WICI_BF16, x.row_stride, x.head_stride};
}

bool tab_ok(const wici_rope_tab* t, int head_dim) {
  return t && aligned(t->cos_t) && aligned(t->sin_t) && t->n_pos >= 1 &&
         t->n_pos <= (int64_t)1 << 24 && t->dim >= 8 && t->dim % 8 == 0 && t->dim <= head_dim &&
         (t->layout == WICI_ROPE_HALF || t->layout == WICI_ROPE_PAIRS);
}
RopeTab tab_of(const wici_rope_tab* t) {
  if (!t) return RopeTab{};
  return RopeTab{t->cos_t, t->sin_t, (int)t->n_pos, t->dim, t->layout};
}

bool geometry_ok(const wici_kv8* c) {
  return c && c->n_pages >= 1 && c->n_kv_heads >= 1 && c->n_kv_heads <= 1024 &&
         (c->head_dim == 64 || c->head_dim == 128) &&
         (c->page == 16 || c->page == 32 || c->page == 64 || c->page == 128);
}
bool batch_shape_ok(const wici_kv8* c, const wici_kv8_batch* b) {
  return b && c->max_pages >= 1 && c->max_pages <= (1 << 24) && b->n_seqs >= 0 &&
         b->n_seqs <= 65535 && b->n_rows >= 0 && b->n_rows <= (1 << 24) && b->max_rows >= 0 &&
         b->max_length >= 0 && (b->row_start || b->n_rows == b->n_seqs);
}
bool empty(const wici_kv8_batch* b) { return b->n_rows == 0 || b->n_seqs == 0; }
bool call_ok(const wici_kv8* c, const wici_kv8_batch* b) {
  return geometry_ok(c) && batch_shape_ok(c, b) && aligned(c->pool) && (c->table || empty(b)) &&
         (b->n_seqs <= 1 || c->table_stride >= c->max_pages) && c->table_stride >= 0 &&
         (b->length || empty(b));
}
Kv8 cache_of(const wici_kv8* c) {
  Kv8 k{};
  k.base = static_cast<char*>(c->pool);
  k.table = c->table;
  k.table_stride = c->table_stride;
  k.n_pages = c->n_pages;
  k.max_pages = c->max_pages;
  k.page_shift = __builtin_ctz((unsigned)c->page);
  k.n_kv = c->n_kv_heads;
  return k;
}
Kv8Rows batch_of(const wici_kv8_batch* b) {
  Kv8Rows r{};
  r.kind = wici::KV8_ARRAYS;
  r.n_seqs = b->n_seqs;
  r.n_rows = b->n_rows;
  r.row_start = b->row_start;
  r.length = b->length;
  return r;
}
// the most rows and positions of a sequence, as the launch plans for them
int most_rows(const wici_kv8_batch* b) {
  return !b->row_start ? 1 : b->max_rows > 0 ? std::min(b->max_rows, b->n_rows) : b->n_rows;
}
int most_length(const wici_kv8* c, const wici_kv8_batch* b) {
  const int64_t cap = (int64_t)c->max_pages * c->page;
  return (int)(b->max_length > 0 ? std::min<int64_t>(b->max_length, cap)
                                 : std::min<int64_t>(cap, 1 << 30));
}

wici_status status(hipError_t e) { return e == hipSuccess ? WICI_OK : WICI_E_HIP; }

}  // namespace

extern "C" {

wici_status wici_rope_table(const wici_rope* rope, int64_t n_pos, float* cos_t, float* sin_t,
                            void* hip_stream) {
  if (!rope || !wici::rope_ok(*rope) || n_pos < 0 || n_pos > (int64_t)1 << 24) return WICI_E_ARG;
  if (n_pos == 0) return WICI_OK;
  if (!cos_t || !sin_t) return WICI_E_ARG;
  OnDeviceOf dev(hip_stream);
  if (!dev.ok()) return WICI_E_HIP;
  return status(wici::launch_rope_table(wici::rope_freqs(*rope), rope->dim / 2, n_pos, cos_t,
                                        sin_t, static_cast<hipStream_t>(hip_stream)));
}

wici_status wici_rope_rows(const wici_rope_tab* rope, int32_t head_dim, int32_t n_rows,
                           int32_t n_heads, const int32_t* positions, wici_head_rows x,
                           wici_head_rows y, void* hip_stream) {
  if ((head_dim != 64 && head_dim != 128) || !tab_ok(rope, head_dim) || n_rows < 0 ||
      n_heads < 1 || n_heads > 1024 || !units_ok(n_rows, n_heads))
    return WICI_E_ARG;
  if (n_rows == 0) return WICI_OK;
  if (!positions || !rows_ok(x, n_heads, head_dim) || !rows_ok(y, n_heads, head_dim))
    return WICI_E_ARG;
  OnDeviceOf dev(hip_stream);
  if (!dev.ok()) return WICI_E_HIP;
  return status(wici::launch_rope_rows(head_dim, rows_of(x), rows_of(y), n_rows, n_heads, positions,
                                       tab_of(rope), static_cast<hipStream_t>(hip_stream)));
}

wici_status wici_kv8_bytes(const wici_kv8* cache, size_t* bytes) {
  if (!geometry_ok(cache) || !bytes) return WICI_E_ARG;
  *bytes = (size_t)cache->n_pages * 2 * cache->n_kv_heads *
           wici::kv8_block_bytes(cache->page, cache->head_dim);
  return WICI_OK;
}

wici_status wici_kv8_append(const wici_kv8* cache, const wici_kv8_batch* batch,
                            const wici_rope_tab* rope, int32_t n_heads, wici_head_rows q,
                            wici_head_rows q_out, wici_head_rows k, wici_head_rows v,
                            void* hip_stream) {
  if (!call_ok(cache, batch) || (rope && !tab_ok(rope, cache->head_dim))) return WICI_E_ARG;
  const int hd = cache->head_dim;
  if (q.data && (!rope || n_heads < 1 || n_heads > 1024)) return WICI_E_ARG;
  if (!units_ok(batch->n_rows, (q.data ? n_heads : 0) + 2 * cache->n_kv_heads)) return WICI_E_ARG;
  if (empty(batch)) return WICI_OK;
  if (!rows_ok(k, cache->n_kv_heads, hd) || !rows_ok(v, cache->n_kv_heads, hd) ||
      (q.data && (!rows_ok(q, n_heads, hd) || !rows_ok(q_out, n_heads, hd))))
    return WICI_E_ARG;
  OnDeviceOf dev(hip_stream);
  if (!dev.ok()) return WICI_E_HIP;
  return status(wici::launch_kv8_append(hd, cache_of(cache), batch_of(batch), tab_of(rope), n_heads,
                                        rows_of(q), rows_of(q_out), 1.0f, rows_of(k), rows_of(v),
                                        static_cast<hipStream_t>(hip_stream)));
}

wici_status wici_kv8_read(const wici_kv8* cache, const wici_kv8_batch* batch, wici_head_rows k,
                          wici_head_rows v, void* hip_stream) {
  if (!call_ok(cache, batch) || !units_ok(batch->n_rows, 2 * cache->n_kv_heads)) return WICI_E_ARG;
  if (empty(batch)) return WICI_OK;
  if ((!k.data && !v.data) || (k.data && !rows_ok(k, cache->n_kv_heads, cache->head_dim)) ||
      (v.data && !rows_ok(v, cache->n_kv_heads, cache->head_dim)))
    return WICI_E_ARG;
  OnDeviceOf dev(hip_stream);
  if (!dev.ok()) return WICI_E_HIP;
  return status(wici::launch_kv8_read(cache->head_dim, cache_of(cache), batch_of(batch), rows_of(k),
                                      rows_of(v), static_cast<hipStream_t>(hip_stream)));
}

wici_status wici_kv8_attend_workspace(const wici_kv8* cache, const wici_kv8_batch* batch,
                                      int32_t n_heads, size_t* bytes) {
  if (!bytes || !geometry_ok(cache) || !batch_shape_ok(cache, batch) || n_heads < 1 ||
      n_heads > 1024 || n_heads % cache->n_kv_heads ||
      (int64_t)batch->n_rows * n_heads > kMostAttended)
    return WICI_E_ARG;
  *bytes = empty(batch) ? 0
                        : 4 * wici::kv8_attn_floats(cache->head_dim, n_heads, cache->n_kv_heads,
                                                    batch->n_seqs, batch->n_rows, most_rows(batch),
                                                    most_length(cache, batch));
  return WICI_OK;
}

wici_status wici_kv8_attend(const wici_kv8* cache, const wici_kv8_batch* batch, int32_t n_heads,
                            float scale, wici_head_rows q, wici_head_rows out, void* workspace,
                            size_t workspace_bytes, void* hip_stream) {
  size_t need = 0;
  if (!call_ok(cache, batch) || !std::isfinite(scale) ||
      wici_kv8_attend_workspace(cache, batch, n_heads, &need) != WICI_OK)
    return WICI_E_ARG;
  if (empty(batch)) return WICI_OK;
  if (!rows_ok(q, n_heads, cache->head_dim) || !rows_ok(out, n_heads, cache->head_dim) ||
      (need && (!aligned(workspace) || workspace_bytes < need)))
    return WICI_E_ARG;
  OnDeviceOf dev(hip_stream);
  if (!dev.ok()) return WICI_E_HIP;
  wici::Kv8Attn a{};
  a.hd = cache->head_dim;
  a.n_q = n_heads;
  a.scale = scale;
  a.q = rows_of(q);
  a.out = rows_of(out);
  a.max_rows = most_rows(batch);
  a.max_length = most_length(cache, batch);
  a.work = static_cast<float*>(workspace);
  return status(wici::launch_kv8_attn(cache_of(cache), batch_of(batch), a,
                                      static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
