// Checks of the arguments that entry points of the 4-bit operators share, on
// the host, before any HIP call.
#pragma once

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

inline bool group_ok(int32_t g) { return g == 32 || g == 64 || g == 128; }

// Tiles of a matrix, 0 where its sizes are not supported.
inline int64_t q4_tiles(int64_t N, int64_t K) {
  if (N < 1 || K < 1 || N > TQ_Q4_MAX_OUT || K > TQ_Q4_MAX_IN) return 0;
  const int64_t tiles = ((N + 15) / 16) * ((K + 127) / 128);
  return tiles < (1 << 24) ? tiles : 0;   // a launch has fewer than 2^32 threads
}

inline tq_status check_q4(const tq_q4_matrix* m, const uint8_t* codes, const uint16_t* params, Q4Dev* d) {
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

inline bool kv_sizes(const tq_kv_cache* c, KvDev* d) {
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

inline tq_status check_kv(const tq_kv_cache* c, KvDev* d) {
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
inline tq_status check_rows(const KvDev& d, const int32_t* seqs, int64_t n_rows, int64_t most) {
  if (n_rows < 1 || n_rows > most) return TQ_ERR_SHAPE;
  if (seqs == nullptr && n_rows > d.n_seqs) return TQ_ERR_SHAPE;
  if (misaligned(seqs, 4)) return TQ_ERR_ALIGN;
  return TQ_OK;
}

inline tq_status check_kv_rows(const tq_kv_rows* r, KvRows* d) {
  if (r == nullptr || r->data == nullptr) return TQ_ERR_NULL;
  if (misaligned(r->data, 2)) return TQ_ERR_ALIGN;
  d->p = r->data;
  d->ts = r->token_stride;
  d->hs = r->head_stride;
  return TQ_OK;
}

// What tq_kv_append and tq_kv_read share.
inline tq_status check_tokens(const tq_kv_cache* cache, int32_t layer, const int32_t* seqs, const int32_t* starts,
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

inline tq_status check_attn(const tq_kv_cache* cache, const tq_kv_attn* a, KvDev* d, AttnCall* c) {
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
