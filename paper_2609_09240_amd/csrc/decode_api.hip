// Host entry points of what a decode step does around its projections, its
// cache and its output head (declared in include/tq.h): argument checks on the
// host, then asynchronous launches on the caller's stream.  Every check runs
// before the first HIP call.

#include "decode_internal.h"
#include "q4_checks.h"

namespace {

using tq::ScopeCall;

// What tq_kv_attention checks, and the scope.
tq_status check_scope(const tq_kv_cache* cache, const tq_kv_attn* a, const tq_kv_scope* scope, KvDev* d, AttnCall* c,
                      ScopeCall* sc) {
  if (scope == nullptr) return TQ_ERR_NULL;
  tq_status st = check_attn(cache, a, d, c);
  if (st != TQ_OK) return st;
  if (scope->sinks < 0 || scope->n_groups < 0 || scope->max_prefix < 0 || scope->max_tail < 0) return TQ_ERR_SHAPE;
  if (scope->n_groups > a->n_rows || (scope->cu_rows == nullptr && scope->n_groups > 1)) return TQ_ERR_SHAPE;
  if (scope->n_groups > 0 && scope->prefix == nullptr) return TQ_ERR_NULL;
  if (misaligned(scope->cu_rows, 4) || misaligned(scope->prefix, 4)) return TQ_ERR_ALIGN;
  *sc = ScopeCall{scope->sinks, scope->n_groups, scope->max_prefix, scope->max_tail, scope->cu_rows, scope->prefix};
  return TQ_OK;
}

tq_status check_logprobs(const tq_logprobs_call* c) {
  if (c == nullptr) return TQ_ERR_NULL;
  if (c->n_rows < 1 || c->n_vocab < 1 || c->n_ids < 0 || c->n_top < 0 || c->n_top > c->n_vocab ||
      c->ld < c->n_vocab)
    return TQ_ERR_SHAPE;
  if (!(c->scale > 0.0f) || !(c->scale <= TQ_LOGPROBS_MAX_SCALE)) return TQ_ERR_SHAPE;
  if (c->n_rows > (1 << 20) || c->n_vocab > (1 << 24) || c->n_ids > TQ_LOGPROBS_MAX_IDS ||
      c->n_top > TQ_LOGPROBS_MAX_TOP || (c->flags != TQ_LOGITS_FP16 && c->flags != TQ_LOGITS_FP32))
    return TQ_ERR_UNSUPPORTED;
  return TQ_OK;
}

// Rows that do not lie on each other.
bool apart(const tq_out_rows& o, int32_t n_tokens, int32_t n_heads) {
  return (n_tokens == 1 || o.token_stride != 0) && (n_heads == 1 || o.head_stride != 0);
}

bool same_rows(const tq_kv_rows& r, const tq_out_rows& o) {
  return r.data == o.data && r.token_stride == o.token_stride && r.head_stride == o.head_stride;
}

}  // namespace

extern "C" {

size_t tq_kv_attention_scope_workspace_bytes(const tq_kv_cache* cache, const tq_kv_attn* a, const tq_kv_scope* scope) {
  KvDev d;
  AttnCall c;
  ScopeCall sc;
  size_t n = 0;
  if (check_scope(cache, a, scope, &d, &c, &sc) != TQ_OK || !tq::kv_scope_plan(d, c, sc, &n)) return 0;
  return n;
}

tq_status tq_kv_attention_scope(const tq_kv_cache* cache, int32_t layer, const tq_kv_attn* a, const tq_kv_scope* scope,
                                void* stream) {
  KvDev d;
  AttnCall c;
  ScopeCall sc;
  tq_status st = check_scope(cache, a, scope, &d, &c, &sc);
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
  if (!tq::kv_scope_plan(d, c, sc, &need)) return TQ_ERR_UNSUPPORTED;
  if (need > 0) {
    if (a->workspace == nullptr) return TQ_ERR_NULL;
    if (a->workspace_bytes < need) return TQ_ERR_SHAPE;
    if (misaligned(a->workspace, 16)) return TQ_ERR_ALIGN;
  }
  return from_hip(tq::launch_kv_attention_scope(d, layer, c, sc, (hipStream_t)stream));
}

tq_status tq_kv_shared_prefix(const tq_kv_cache* cache, const int32_t* seqs, const int32_t* cu_rows, int32_t n_groups,
                              int32_t n_rows, int32_t* prefix, void* stream) {
  KvDev d;
  tq_status st = check_kv(cache, &d);
  if (st != TQ_OK) return st;
  if ((st = check_rows(d, seqs, n_rows, 65535)) != TQ_OK) return st;
  if (n_groups < 1 || n_groups > n_rows || (cu_rows == nullptr && n_groups > 1)) return TQ_ERR_SHAPE;
  if (prefix == nullptr) return TQ_ERR_NULL;
  if (misaligned(cu_rows, 4) || misaligned(prefix, 4)) return TQ_ERR_ALIGN;
  return from_hip(tq::launch_kv_shared_prefix(d, seqs, cu_rows, n_groups, n_rows, prefix, (hipStream_t)stream));
}

tq_status tq_rope(const tq_rope_call* c, void* stream) {
  if (c == nullptr) return TQ_ERR_NULL;
  if (c->n_tokens < 1 || c->n_heads < 1 || c->n_kv_heads < 0 || c->rot < 2 || c->rot % 2 != 0 ||
      c->rot > c->head_dim || c->n_axes < 1 || !isfinite(c->scale))
    return TQ_ERR_SHAPE;
  if (c->head_dim > TQ_ROPE_MAX_DIM || c->n_axes > TQ_ROPE_MAX_AXES ||
      (c->flags & ~(TQ_ROPE_ADJACENT | TQ_ROPE_INVERSE)) != 0 || c->n_tokens > TQ_ROPE_MAX_TOKENS ||
      c->n_heads > TQ_ROPE_MAX_HEADS || c->n_kv_heads > TQ_ROPE_MAX_HEADS)
    return TQ_ERR_UNSUPPORTED;
  if (c->positions == nullptr || c->freq == nullptr || c->q.data == nullptr || c->q_out.data == nullptr)
    return TQ_ERR_NULL;
  if (c->n_kv_heads > 0 && (c->k.data == nullptr || c->k_out.data == nullptr)) return TQ_ERR_NULL;
  if (misaligned(c->positions, 4) || misaligned(c->freq, 4) || misaligned(c->q.data, 2) || misaligned(c->q_out.data, 2) ||
      misaligned(c->k.data, 2) || misaligned(c->k_out.data, 2))
    return TQ_ERR_ALIGN;
  if (!apart(c->q_out, c->n_tokens, c->n_heads) || (c->n_kv_heads > 0 && !apart(c->k_out, c->n_tokens, c->n_kv_heads)))
    return TQ_ERR_SHAPE;
  // An output that starts where its input does is the input.
  if ((c->q.data == c->q_out.data && !same_rows(c->q, c->q_out)) ||
      (c->n_kv_heads > 0 && c->k.data == c->k_out.data && !same_rows(c->k, c->k_out)))
    return TQ_ERR_SHAPE;
  return from_hip(tq::launch_rope(*c, (hipStream_t)stream));
}

size_t tq_logprobs_workspace_bytes(const tq_logprobs_call* c) {
  return check_logprobs(c) == TQ_OK ? tq::logprobs_workspace_bytes(*c) : 0;
}

tq_status tq_logprobs(const tq_logprobs_call* c, void* stream) {
  const tq_status st = check_logprobs(c);
  if (st != TQ_OK) return st;
  if (c->logits == nullptr || (c->n_ids > 0 && (c->ids == nullptr || c->logp == nullptr)) ||
      (c->n_top > 0 && (c->top_ids == nullptr || c->top_logp == nullptr)))
    return TQ_ERR_NULL;
  if (misaligned(c->logits, c->flags == TQ_LOGITS_FP32 ? 4 : 2) || misaligned(c->ids, 4) || misaligned(c->logp, 4) ||
      misaligned(c->entropy, 4) || misaligned(c->top_ids, 4) || misaligned(c->top_logp, 4) || misaligned(c->d_err, 4))
    return TQ_ERR_ALIGN;
  const size_t need = tq::logprobs_workspace_bytes(*c);
  if (need > 0) {
    if (c->workspace == nullptr) return TQ_ERR_NULL;
    if (c->workspace_bytes < need) return TQ_ERR_SHAPE;
    if (misaligned(c->workspace, 16)) return TQ_ERR_ALIGN;
  }
  return from_hip(tq::launch_logprobs(*c, (hipStream_t)stream));
}

}  // extern "C"
