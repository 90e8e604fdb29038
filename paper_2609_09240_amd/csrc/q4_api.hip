// Host entry points of the 4-bit operators (declared in include/tq.h):
// argument checks on the host, then asynchronous launches on the caller's
// stream.  Every check runs before the first HIP call.

#include <math.h>
#include <stdint.h>

#include "q4_internal.h"

namespace {

using tq::AttnCall;
using tq::KvDev;
using tq::KvRows;
using tq::Q4Dev;

inline bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

inline tq_status from_hip(hipError_t e) { return e == hipSuccess ? TQ_OK : TQ_ERR_HIP; }

bool group_ok(int32_t g) { return g == 32 || g == 64 || g == 128; }

// Tiles of a matrix, 0 where its sizes are not supported.
int64_t q4_tiles(int64_t N, int64_t K) {
  if (N < 1 || K < 1 || N > TQ_Q4_MAX_OUT || K > TQ_Q4_MAX_IN) return 0;
  const int64_t tiles = ((N + 15) / 16) * ((K + 127) / 128);
  return tiles < (1 << 24) ? tiles : 0;   // a launch has fewer than 2^32 threads
}

tq_status check_q4(const tq_q4_matrix* m, const uint8_t* codes, const uint16_t* params, Q4Dev* d) {
  if (m == nullptr) return TQ_ERR_NULL;
  if (!group_ok(m->group)) return TQ_ERR_UNSUPPORTED;
  if (m->reserved != 0 || m->n_out < 1 || m->n_in < 1) return TQ_ERR_SHAPE;
  if (q4_tiles(m->n_out, m->n_in) == 0) return TQ_ERR_UNSUPPORTED;
  if (codes == nullptr || params == nullptr) return TQ_ERR_NULL;
  if (misaligned(codes, 16) || misaligned(params, 16)) return TQ_ERR_ALIGN;
  d->codes = codes;
  d->params = params;
  d->n_out = (int32_t)m->n_out;
  d->n_in = (int32_t)m->n_in;
  d->group = m->group;
  return TQ_OK;
}

bool kv_sizes(const tq_kv_cache* c, KvDev* d) {
  if (c->n_layers < 1 || c->n_layers > 65535 || c->n_kv_heads < 1 || c->n_kv_heads > 1024) return false;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return false;
  if (!group_ok(c->group) || c->group > c->head_dim) return false;
  int shift = 5;
  while (shift < 10 && (1 << shift) != c->page_size) ++shift;
  if ((1 << shift) != c->page_size) return false;
  d->n_layers = c->n_layers;
  d->H = c->n_kv_heads;
  d->D = c->head_dim;
  d->G = c->group;
  d->page_size = c->page_size;
  d->page_shift = shift;
  d->page_bytes = (int64_t)d->H * (c->page_size / 32) * tq::kv_record_bytes(d->D, d->G);
  return true;
}

tq_status check_kv(const tq_kv_cache* c, KvDev* d) {
  if (c == nullptr) return TQ_ERR_NULL;
  if (c->reserved != 0 || c->n_seqs < 1 || c->max_pages < 1 || c->n_pages < 1) return TQ_ERR_SHAPE;
  if (!kv_sizes(c, d) || c->max_pages > TQ_KV_MAX_PAGES || c->n_pages > (1 << 30)) return TQ_ERR_UNSUPPORTED;
  if (c->data == nullptr || c->pages == nullptr || c->lens == nullptr || c->refs == nullptr) return TQ_ERR_NULL;
  if (misaligned(c->data, 16) || misaligned(c->pages, 4) || misaligned(c->lens, 4) || misaligned(c->refs, 4))
    return TQ_ERR_ALIGN;
  d->data = c->data;
  d->pages = c->pages;
  d->lens = c->lens;
  d->refs = c->refs;
  d->n_seqs = c->n_seqs;
  d->max_pages = c->max_pages;
  d->n_pages = (int32_t)c->n_pages;
  d->layer_bytes = c->n_pages * d->page_bytes;
  return TQ_OK;
}

// Rows of a call: n_rows of them, seqs NULL only where slot i is row i.
tq_status check_rows(const KvDev& d, const int32_t* seqs, int64_t n_rows, int64_t most) {
  if (n_rows < 1 || n_rows > most) return TQ_ERR_SHAPE;
  if (seqs == nullptr && n_rows > d.n_seqs) return TQ_ERR_SHAPE;
  if (misaligned(seqs, 4)) return TQ_ERR_ALIGN;
  return TQ_OK;
}

tq_status check_kv_rows(const tq_kv_rows* r, KvRows* d) {
  if (r == nullptr || r->data == nullptr) return TQ_ERR_NULL;
  if (misaligned(r->data, 2)) return TQ_ERR_ALIGN;
  d->p = r->data;
  d->ts = r->token_stride;
  d->hs = r->head_stride;
  return TQ_OK;
}

// What tq_kv_append and tq_kv_read share.
tq_status check_tokens(const tq_kv_cache* cache, int32_t layer, const int32_t* seqs, const int32_t* starts,
                       const int32_t* cu_new, int32_t n_rows, int32_t n_tokens, int32_t max_new, KvDev* d) {
  tq_status st = check_kv(cache, d);
  if (st != TQ_OK) return st;
  if (layer < 0 || layer >= d->n_layers) return TQ_ERR_SHAPE;
  if ((st = check_rows(*d, seqs, n_rows, 65535)) != TQ_OK) return st;
  if (n_tokens < 1 || max_new < 1 || max_new > (1 << 26)) return TQ_ERR_SHAPE;
  if (starts == nullptr) return TQ_ERR_NULL;
  if (misaligned(starts, 4) || misaligned(cu_new, 4)) return TQ_ERR_ALIGN;
  return TQ_OK;
}

tq_status check_attn(const tq_kv_cache* cache, const tq_kv_attn* a, KvDev* d, AttnCall* c) {
  if (cache == nullptr || a == nullptr) return TQ_ERR_NULL;
  tq_status st = check_kv(cache, d);
  if (st != TQ_OK) return st;
  if ((st = check_rows(*d, a->seqs, a->n_rows, 65535)) != TQ_OK) return st;
  if (a->n_tokens < 1 || a->max_q < 1 || a->max_len < 0 || a->window < 0) return TQ_ERR_SHAPE;
  if (a->n_heads < 1 || a->n_heads % d->H != 0) return TQ_ERR_SHAPE;
  if (a->flags != TQ_OUT_FP16 && a->flags != TQ_OUT_FP32) return TQ_ERR_UNSUPPORTED;
  if (!isfinite(a->scale)) return TQ_ERR_SHAPE;
  if (a->n_heads > TQ_KV_MAX_HEADS || (int64_t)a->n_tokens * a->n_heads > INT32_MAX) return TQ_ERR_UNSUPPORTED;
  c->n_rows = a->n_rows;
  c->n_tokens = a->n_tokens;
  c->max_q = a->max_q < a->n_tokens ? a->max_q : a->n_tokens;
  c->n_heads = a->n_heads;
  c->max_len = a->max_len;
  c->window = a->window;
  c->scale = a->scale;
  c->out_f32 = a->flags == TQ_OUT_FP32;
  c->seqs = a->seqs;
  c->cu = a->cu_q;
  return TQ_OK;
}

}  // namespace

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
