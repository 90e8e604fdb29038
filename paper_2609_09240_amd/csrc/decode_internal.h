// Launchers behind the entry points of decode_api.hip, which has checked
// their arguments.
#pragma once

#include "q4_internal.h"

namespace tq {

// ---- Attention with sinks or shared prefixes (kvscope.hip).
struct ScopeCall {
  int32_t sinks, n_groups, max_prefix, max_tail;
  const int32_t* cu_rows;
  const int32_t* prefix;
};
// false where the launch would not fit a grid.
bool kv_scope_plan(const KvDev& c, const AttnCall& a, const ScopeCall& sc, size_t* ws_bytes);
hipError_t launch_kv_attention_scope(const KvDev& c, int layer, const AttnCall& a, const ScopeCall& sc, hipStream_t s);
hipError_t launch_kv_shared_prefix(const KvDev& c, const int32_t* seqs, const int32_t* cu_rows, int n_groups,
                                   int n_rows, int32_t* prefix, hipStream_t s);

// ---- Rotary positions (rope.hip).
hipError_t launch_rope(const tq_rope_call& c, hipStream_t s);

// ---- Log probabilities (logprobs.hip).
size_t logprobs_workspace_bytes(const tq_logprobs_call& c);
hipError_t launch_logprobs(const tq_logprobs_call& c, hipStream_t s);

}  // namespace tq
