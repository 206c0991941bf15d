// kv4_api.cu — entry points of the paged 4-bit cache: argument checks and launches.
#include "checks.h"
#include "kernels.h"
#include "kv4.cuh"

using namespace semkv;

namespace {

semkv_status from_cuda(cudaError_t e) { return e == cudaSuccess ? SEMKV_OK : SEMKV_ECUDA; }

semkv_status check_kv4(const semkv_kv4_cache* c, Kv4Cache& to) {
  if (!c) return SEMKV_EINVAL;
  if (c->layers < 1 || c->kv_heads < 1 || c->num_pages < 1 || c->max_seqs < 1 || c->max_pages < 1)
    return SEMKV_EINVAL;
  if (c->head_dim != 64 && c->head_dim != 128) return SEMKV_EUNSUPPORTED;
  if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128)
    return SEMKV_EUNSUPPORTED;
  // token positions are 32-bit inside the kernels
  if ((int64_t)c->max_pages * c->page_tokens > (int64_t)1 << 30) return SEMKV_EUNSUPPORTED;
  if (!c->pages || !c->table || !c->length || !c->refs) return SEMKV_EINVAL;
  if (!aligned(c->pages, 16) || !aligned(c->refs, 16) || !aligned(c->table, 4) || !aligned(c->length, 4) ||
      !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4) || !aligned(c->dev_error, 4))
    return SEMKV_EALIGN;
  to.layers = c->layers;
  to.H = c->kv_heads;
  to.D = c->head_dim;
  to.P = c->page_tokens;
  to.page_shift = c->page_tokens == 16 ? 4 : c->page_tokens == 32 ? 5 : c->page_tokens == 64 ? 6 : 7;
  to.num_pages = c->num_pages;
  to.max_seqs = c->max_seqs;
  to.max_pages = c->max_pages;
  to.pages = c->pages;
  to.k_scale = c->k_scale;
  to.v_scale = c->v_scale;
  to.table = c->table;
  to.length = c->length;
  to.refs = c->refs;
  to.err = c->dev_error;
  return SEMKV_OK;
}

semkv_status check_list(int32_t n, const int32_t* seqs) {
  if (n < 0) return SEMKV_EINVAL;
  if (n > SEMKV_KV4_MAX_SEQS) return SEMKV_EUNSUPPORTED;
  return aligned(seqs, 4) ? SEMKV_OK : SEMKV_EALIGN;
}

semkv_status check_kv4_batch(const semkv_kv4_batch* b, bool start, Kv4Batch& to) {
  if (!b || b->total < 0 || b->max_count < (b->total > 0)) return SEMKV_EINVAL;
  const semkv_status s = check_list(b->n, b->seqs);
  if (s != SEMKV_OK) return s;
  if ((!b->cu && b->total < b->n) || (start && !b->start && b->n > 0)) return SEMKV_EINVAL;
  // row indices are 32-bit inside the kernels
  if (b->total > 1 << 30) return SEMKV_EUNSUPPORTED;
  if (!aligned(b->cu, 4) || !aligned(b->start, 4)) return SEMKV_EALIGN;
  to.n = b->n;
  to.total = b->total;
  to.max_count = b->max_count;
  to.seqs = b->seqs;
  to.cu = b->cu;
  to.start = b->start;
  return SEMKV_OK;
}

semkv_status check_ws(const void* ws, size_t bytes, size_t want) {
  return !ws || !aligned(ws, 16) || bytes < want ? SEMKV_EWORKSPACE : SEMKV_OK;
}

semkv_status rows(const semkv_kv4_cache* cache, const semkv_kv4_batch* batch, bool write, int32_t layer, int32_t dtype,
                  void* k, int64_t k_stride, void* v, int64_t v_stride, void* stream) {
  Kv4Cache c;
  Kv4Batch b;
  semkv_status s = check_kv4(cache, c);
  if (s != SEMKV_OK) return s;
  s = check_kv4_batch(batch, true, b);
  if (s != SEMKV_OK) return s;
  if ((b.total > 0 && (!k || !v)) || layer < 0 || layer >= c.layers) return SEMKV_EINVAL;
  if (dtype != SEMKV_F16 && dtype != SEMKV_BF16) return SEMKV_EUNSUPPORTED;
  if (k_stride < (int64_t)c.H * c.D || v_stride < (int64_t)c.H * c.D) return SEMKV_EINVAL;
  if (!aligned(k, 16) || !aligned(v, 16) || k_stride % 8 || v_stride % 8) return SEMKV_EALIGN;
  if (b.n == 0 || b.total == 0) return SEMKV_OK;
  const int sms = device_sm_count();
  if (sms <= 0) return SEMKV_ECUDA;
  return from_cuda(launch_kv4_rows(c, b, write, layer, dtype, k, k_stride, v, v_stride, sms, (cudaStream_t)stream));
}

}  // namespace

extern "C" {

size_t semkv_kv4_tile_bytes(int32_t head_dim) {
  return head_dim == 64 || head_dim == 128 ? (size_t)kv4_tile_bytes(head_dim) : 0;
}

size_t semkv_kv4_pages_workspace_bytes(const semkv_kv4_cache* cache, int32_t n, int32_t tokens) {
  Kv4Cache c;
  if (check_kv4(cache, c) != SEMKV_OK || check_list(n, nullptr) != SEMKV_OK) return 0;
  return kv4_pages_workspace(c, n, tokens, tokens >= 0);
}

semkv_status semkv_kv4_reserve(const semkv_kv4_cache* cache, const semkv_kv4_batch* batch, void* ws, size_t ws_bytes,
                               void* stream) {
  const TraceRange trace("semkv_kv4_reserve");
  Kv4Cache c;
  Kv4Batch b;
  semkv_status s = check_kv4(cache, c);
  if (s != SEMKV_OK) return s;
  s = check_kv4_batch(batch, true, b);
  if (s != SEMKV_OK) return s;
  if (b.n == 0) return SEMKV_OK;
  s = check_ws(ws, ws_bytes, kv4_pages_workspace(c, b.n, 0, false));
  if (s != SEMKV_OK) return s;
  const int sms = device_sm_count();
  if (sms <= 0) return SEMKV_ECUDA;
  return from_cuda(launch_kv4_reserve(c, b, ws, sms, (cudaStream_t)stream));
}

semkv_status semkv_kv4_write(const semkv_kv4_cache* cache, const semkv_kv4_batch* batch, int32_t layer, int32_t dtype,
                             const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* stream) {
  const TraceRange trace("semkv_kv4_write");
  return rows(cache, batch, true, layer, dtype, const_cast<void*>(k), k_stride, const_cast<void*>(v), v_stride, stream);
}

semkv_status semkv_kv4_read(const semkv_kv4_cache* cache, const semkv_kv4_batch* batch, int32_t layer, int32_t dtype,
                            void* k_out, void* v_out, void* stream) {
  const TraceRange trace("semkv_kv4_read");
  const int64_t row = cache ? (int64_t)cache->kv_heads * cache->head_dim : 0;
  return rows(cache, batch, false, layer, dtype, k_out, row, v_out, row, stream);
}

size_t semkv_kv4_attention_workspace_bytes(const semkv_kv4_cache* cache, const semkv_kv4_batch* batch, int32_t q_heads) {
  Kv4Cache c;
  Kv4Batch b;
  if (check_kv4(cache, c) != SEMKV_OK || check_kv4_batch(batch, false, b) != SEMKV_OK) return 0;
  if (q_heads < 1 || q_heads % c.H) return 0;
  const int sms = device_sm_count();
  return sms > 0 ? kv4_attention_workspace(c, b, q_heads, sms) : 0;
}

semkv_status semkv_kv4_attention(const semkv_kv4_cache* cache, const semkv_kv4_batch* batch, int32_t layer, int32_t dtype,
                                 const void* q, int64_t q_stride, int32_t q_heads, void* out, float* lse,
                                 float softmax_scale, int32_t window, void* ws, size_t ws_bytes, void* stream) {
  const TraceRange trace("semkv_kv4_attention");
  Kv4Cache c;
  Kv4Batch b;
  semkv_status s = check_kv4(cache, c);
  if (s != SEMKV_OK) return s;
  s = check_kv4_batch(batch, false, b);
  if (s != SEMKV_OK) return s;
  if ((b.total > 0 && (!q || !out)) || layer < 0 || layer >= c.layers || window < 0) return SEMKV_EINVAL;
  if (q_heads < 1 || q_heads % c.H) return SEMKV_EINVAL;
  if (dtype != SEMKV_F16 && dtype != SEMKV_BF16) return SEMKV_EUNSUPPORTED;
  // row indices of a sequence are 32-bit inside the kernels
  if ((int64_t)b.max_count * (q_heads / c.H) > (int64_t)1 << 30) return SEMKV_EUNSUPPORTED;
  if (q_stride < (int64_t)q_heads * c.D) return SEMKV_EINVAL;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4) || q_stride % 8) return SEMKV_EALIGN;
  if (b.n == 0 || b.total == 0) return SEMKV_OK;
  const int sms = device_sm_count();
  if (sms <= 0) return SEMKV_ECUDA;
  s = check_ws(ws, ws_bytes, kv4_attention_workspace(c, b, q_heads, sms));
  if (s != SEMKV_OK) return s;
  return from_cuda(launch_kv4_attention(c, b, layer, dtype, q, q_stride, q_heads, out, lse, softmax_scale, window, ws, sms,
                                        (cudaStream_t)stream));
}

semkv_status semkv_kv4_fork(const semkv_kv4_cache* cache, int32_t n, const int32_t* src, const int32_t* dst, void* stream) {
  const TraceRange trace("semkv_kv4_fork");
  Kv4Cache c;
  semkv_status s = check_kv4(cache, c);
  if (s != SEMKV_OK) return s;
  s = check_list(n, src);
  if (s != SEMKV_OK) return s;
  if (n > 0 && (!src || !dst)) return SEMKV_EINVAL;
  if (!aligned(dst, 4)) return SEMKV_EALIGN;
  if (n == 0) return SEMKV_OK;
  return from_cuda(launch_kv4_fork(c, n, src, dst, (cudaStream_t)stream));
}

semkv_status semkv_kv4_free(const semkv_kv4_cache* cache, int32_t n, const int32_t* seqs, void* stream) {
  const TraceRange trace("semkv_kv4_free");
  Kv4Cache c;
  semkv_status s = check_kv4(cache, c);
  if (s != SEMKV_OK) return s;
  s = check_list(n, seqs);
  if (s != SEMKV_OK || n == 0) return s;
  return from_cuda(launch_kv4_free(c, n, seqs, (cudaStream_t)stream));
}

semkv_status semkv_kv4_compact(const semkv_kv4_cache* cache, int32_t n, const int32_t* seqs, const uint8_t* keep,
                               int32_t tokens, void* ws, size_t ws_bytes, void* stream) {
  const TraceRange trace("semkv_kv4_compact");
  Kv4Cache c;
  semkv_status s = check_kv4(cache, c);
  if (s != SEMKV_OK) return s;
  s = check_list(n, seqs);
  if (s != SEMKV_OK) return s;
  if (tokens < 0 || (n > 0 && tokens > 0 && !keep)) return SEMKV_EINVAL;
  if (n == 0) return SEMKV_OK;
  s = check_ws(ws, ws_bytes, kv4_pages_workspace(c, n, tokens, true));
  if (s != SEMKV_OK) return s;
  const int sms = device_sm_count();
  if (sms <= 0) return SEMKV_ECUDA;
  return from_cuda(launch_kv4_compact(c, n, seqs, keep, tokens, ws, sms, (cudaStream_t)stream));
}

}  // extern "C"
