// Host entry points of the 4-bit operators (declared in include/tq.h):
// argument checks on the host, then asynchronous launches on the caller's
// stream.  Every check runs before the first HIP call.

#include "q4_checks.h"

extern "C" {

size_t tq_q4_code_bytes(int64_t n_out, int64_t n_in) { return (size_t)q4_tiles(n_out, n_in) * 1024; }

size_t tq_q4_param_bytes(int64_t n_out, int64_t n_in, int32_t group) {
  return group_ok(group) ? (size_t)q4_tiles(n_out, n_in) * (128 / group) * 64 : 0;
}

tq_status tq_q4_quantize(const uint16_t* w, int64_t ldw, const tq_q4_matrix* m, uint8_t* codes, uint16_t* params,
                         void* stream) {
  Q4Dev d;
  tq_status st = check_q4(m, codes, params, &d);
  if (st != TQ_OK) return st;
  if (w == nullptr) return TQ_ERR_NULL;
  if (ldw < m->n_in) return TQ_ERR_SHAPE;
  if (misaligned(w, 2)) return TQ_ERR_ALIGN;
  return from_hip(tq::launch_q4_quantize(w, ldw, d, codes, params, (hipStream_t)stream));
}

tq_status tq_q4_unpack_fp16(const tq_q4_matrix* m, uint16_t* w, void* stream) {
  if (m == nullptr) return TQ_ERR_NULL;
  Q4Dev d;
  tq_status st = check_q4(m, m->codes, m->params, &d);
  if (st != TQ_OK) return st;
  if (w == nullptr) return TQ_ERR_NULL;
  if (misaligned(w, 2)) return TQ_ERR_ALIGN;
  return from_hip(tq::launch_q4_unpack(d, w, (hipStream_t)stream));
}

size_t tq_q4_workspace_bytes(const tq_q4_matrix* m, int32_t B) {
  Q4Dev d;
  if (m == nullptr || B < 1 || B > TQ_Q4_MAX_BATCH || check_q4(m, m->codes, m->params, &d) != TQ_OK) return 0;
  return tq::q4_workspace_bytes(d, B);
}

tq_status tq_q4_gemm(const tq_q4_matrix* m, const uint16_t* X, int64_t ldx, int32_t B, void* Y, int32_t flags,
                     void* workspace, size_t workspace_bytes, void* stream) {
  if (m == nullptr) return TQ_ERR_NULL;
  Q4Dev d;
  tq_status st = check_q4(m, m->codes, m->params, &d);
  if (st != TQ_OK) return st;
  if (flags != TQ_OUT_FP16 && flags != TQ_OUT_FP32) return TQ_ERR_UNSUPPORTED;
  if (X == nullptr || Y == nullptr) return TQ_ERR_NULL;
  if (B < 1 || B > TQ_Q4_MAX_BATCH || ldx < m->n_in) return TQ_ERR_SHAPE;
  if (misaligned(X, 2) || misaligned(Y, 4)) return TQ_ERR_ALIGN;
  if (workspace != nullptr) {
    if (workspace_bytes < tq::q4_workspace_bytes(d, B)) return TQ_ERR_SHAPE;
    if (misaligned(workspace, 16)) return TQ_ERR_ALIGN;
  }
  return from_hip(tq::launch_q4_gemm(d, X, ldx, B, Y, flags == TQ_OUT_FP32, workspace, (hipStream_t)stream));
}

size_t tq_kv_page_bytes(const tq_kv_cache* cache) {
  KvDev d;
  return cache != nullptr && kv_sizes(cache, &d) ? (size_t)d.page_bytes : 0;
}

tq_status tq_kv_extend(const tq_kv_cache* cache, const int32_t* seqs, const int32_t* cu_new, int32_t n_rows,
                       int32_t* starts, int32_t* d_err, void* stream) {
  KvDev d;
  tq_status st = check_kv(cache, &d);
  if (st != TQ_OK) return st;
  if ((st = check_rows(d, seqs, n_rows, TQ_KV_MAX_ROWS)) != TQ_OK) return st;
  if (starts == nullptr) return TQ_ERR_NULL;
  if (misaligned(starts, 4) || misaligned(cu_new, 4) || misaligned(d_err, 4)) return TQ_ERR_ALIGN;
  return from_hip(tq::launch_kv_extend(d, seqs, cu_new, n_rows, starts, d_err, (hipStream_t)stream));
}

tq_status tq_kv_free(const tq_kv_cache* cache, const int32_t* seqs, int32_t n_rows, int32_t* d_err, void* stream) {
  KvDev d;
  tq_status st = check_kv(cache, &d);
  if (st != TQ_OK) return st;
  if ((st = check_rows(d, seqs, n_rows, TQ_KV_MAX_ROWS)) != TQ_OK) return st;
  if (misaligned(d_err, 4)) return TQ_ERR_ALIGN;
  return from_hip(tq::launch_kv_free(d, seqs, n_rows, d_err, (hipStream_t)stream));
}

size_t tq_kv_workspace_bytes(const tq_kv_cache* cache, int32_t n_rows) {
  if (cache == nullptr || n_rows < 0 || n_rows > TQ_KV_MAX_ROWS || cache->n_pages < 1 ||
      cache->n_pages > (1 << 30))
    return 0;
  KvDev d;
  d.n_pages = (int32_t)cache->n_pages;
  return tq::kv_workspace_bytes(d, n_rows);
}

tq_status tq_kv_fork(const tq_kv_cache* cache, const int32_t* parents, const int32_t* children, int32_t n_rows,
                     int32_t* d_err, void* workspace, size_t workspace_bytes, void* stream) {
  KvDev d;
  tq_status st = check_kv(cache, &d);
  if (st != TQ_OK) return st;
  if (n_rows < 1 || n_rows > TQ_KV_MAX_ROWS) return TQ_ERR_SHAPE;
  if (parents == nullptr || children == nullptr || workspace == nullptr) return TQ_ERR_NULL;
  if (workspace_bytes < tq::kv_workspace_bytes(d, n_rows)) return TQ_ERR_SHAPE;
  if (misaligned(parents, 4) || misaligned(children, 4) || misaligned(d_err, 4) || misaligned(workspace, 16))
    return TQ_ERR_ALIGN;
  return from_hip(tq::launch_kv_fork(d, parents, children, n_rows, d_err, workspace, (hipStream_t)stream));
}

tq_status tq_kv_compact(const tq_kv_cache* cache, int32_t* n_live, void* workspace, size_t workspace_bytes,
                        void* stream) {
  KvDev d;
  tq_status st = check_kv(cache, &d);
  if (st != TQ_OK) return st;
  if (workspace == nullptr) return TQ_ERR_NULL;
  if (workspace_bytes < tq::kv_workspace_bytes(d, 0)) return TQ_ERR_SHAPE;
  if (misaligned(n_live, 4) || misaligned(workspace, 16)) return TQ_ERR_ALIGN;
  return from_hip(tq::launch_kv_compact(d, n_live, workspace, (hipStream_t)stream));
}

tq_status tq_kv_copy_pages(const tq_kv_cache* cache, const int32_t* src, const int32_t* dst, int32_t n,
                           int32_t* d_err, void* stream) {
  KvDev d;
  tq_status st = check_kv(cache, &d);
  if (st != TQ_OK) return st;
  if (n < 1 || n > 65535) return TQ_ERR_SHAPE;
  if (src == nullptr || dst == nullptr) return TQ_ERR_NULL;
  if (misaligned(src, 4) || misaligned(dst, 4) || misaligned(d_err, 4)) return TQ_ERR_ALIGN;
  return from_hip(tq::launch_kv_copy_pages(d, src, dst, n, d_err, (hipStream_t)stream));
}

tq_status tq_kv_append(const tq_kv_cache* cache, int32_t layer, const int32_t* seqs, const int32_t* starts,
                       const int32_t* cu_new, int32_t n_rows, int32_t n_tokens, int32_t max_new, const tq_kv_rows* k,
                       const tq_kv_rows* v, int32_t* d_err, void* stream) {
  KvDev d;
  tq_status st = check_tokens(cache, layer, seqs, starts, cu_new, n_rows, n_tokens, max_new, &d);
  if (st != TQ_OK) return st;
  KvRows kr, vr;
  if ((st = check_kv_rows(k, &kr)) != TQ_OK || (st = check_kv_rows(v, &vr)) != TQ_OK) return st;
  if (misaligned(d_err, 4)) return TQ_ERR_ALIGN;
  return from_hip(tq::launch_kv_append(d, layer, seqs, starts, cu_new, n_rows, n_tokens, max_new, kr, vr, d_err,
                                       (hipStream_t)stream));
}

tq_status tq_kv_read(const tq_kv_cache* cache, int32_t layer, const int32_t* seqs, const int32_t* starts,
                     const int32_t* cu_new, int32_t n_rows, int32_t n_tokens, int32_t max_new, uint16_t* k_out,
                     uint16_t* v_out, void* stream) {
  KvDev d;
  tq_status st = check_tokens(cache, layer, seqs, starts, cu_new, n_rows, n_tokens, max_new, &d);
  if (st != TQ_OK) return st;
  if (k_out == nullptr || v_out == nullptr) return TQ_ERR_NULL;
  if (misaligned(k_out, 16) || misaligned(v_out, 16)) return TQ_ERR_ALIGN;
  return from_hip(tq::launch_kv_read(d, layer, seqs, starts, cu_new, n_rows, n_tokens, max_new, k_out, v_out,
                                     (hipStream_t)stream));
}

size_t tq_kv_attention_workspace_bytes(const tq_kv_cache* cache, const tq_kv_attn* a) {
  KvDev d;
  AttnCall c;
  size_t n = 0;
  if (check_attn(cache, a, &d, &c) != TQ_OK || !tq::kv_attention_plan(d, c, &n)) return 0;
  return n;
}

tq_status tq_kv_attention(const tq_kv_cache* cache, int32_t layer, const tq_kv_attn* a, void* stream) {
  KvDev d;
  AttnCall c;
  tq_status st = check_attn(cache, a, &d, &c);
  if (st != TQ_OK) return st;
  if (layer < 0 || layer >= d.n_layers) return TQ_ERR_SHAPE;
  if ((st = check_kv_rows(&a->q, &c.q)) != TQ_OK) return st;
  if (a->o == nullptr) return TQ_ERR_NULL;
  if (misaligned(a->o, 16) || misaligned(a->lse, 4) || misaligned(a->seqs, 4) || misaligned(a->cu_q, 4))
    return TQ_ERR_ALIGN;
  c.o = a->o;
  c.lse = a->lse;
  c.ws = a->workspace;
  size_t need;
  if (!tq::kv_attention_plan(d, c, &need)) return TQ_ERR_UNSUPPORTED;
  if (need > 0) {
    if (a->workspace == nullptr) return TQ_ERR_NULL;
    if (a->workspace_bytes < need) return TQ_ERR_SHAPE;
    if (misaligned(a->workspace, 16)) return TQ_ERR_ALIGN;
  }
  return from_hip(tq::launch_kv_attention(d, layer, c, (hipStream_t)stream));
}

}  // extern "C"
