// Attention of every row over its own tokens (the kernel and its figures:
// kvattn_kernel.h).

#include "kvattn_kernel.h"

namespace tq {
namespace {

bool plan(const KvDev& c, const AttnCall& a, Plan* p) {
  int64_t len = length_hint(c, a);
  if (a.window > 0 && len > (int64_t)a.window + a.max_q) len = (int64_t)a.window + a.max_q;
  return plan(c, (int64_t)a.max_q * (a.n_heads / c.H), a.n_rows, len, p);
}

}  // namespace

bool kv_attention_plan(const KvDev& c, const AttnCall& a, size_t* ws_bytes) {
  Plan p;
  if (!plan(c, a, &p)) return false;
  *ws_bytes = p.shares > 0 ? kCountBytes + part_bytes(c, p) : 0;
  return true;
}

hipError_t launch_kv_attention(const KvDev& c, int layer, const AttnCall& call, hipStream_t s) {
  Plan p;
  if (!plan(c, call, &p)) return hipErrorInvalidValue;
  Args a;
  fill(a, c, layer, call, p);
  const dim3 grid = p.shares ? dim3(p.shares) : dim3(a.H, a.n_rows, p.tiles);
  return with_sizes(c, [&](auto D, auto G) { kv_attn_kernel<D(), G(), kPlain><<<grid, 64 * kWaves, 0, s>>>(a); });
}

}  // namespace tq
