// Attention over the 4-bit paged cache with sinks beside a window, and of
// rows that share the pages of a prefix (gfx950).
//
// Sinks: the records of a tile are those of its window and, in front of them,
// the first ones of the slot; masks in the records where they end.
//
// Shared prefixes, two launches.  The softmax over all tokens of a row is joined
// from those over any parts of them: with m the largest logit of a part, l = sum
// exp(s - m) and y = sum exp(s - m) v,
//     o = sum_parts exp(m - M) y / sum_parts exp(m - M) l,   M = max of the m.
// The first launch takes the queries of all rows of a group as the rows of its
// tiles, over the shared records, and leaves (y, m, l) of every query and head.
// The second one is a row over its own records, which takes them up when it
// stores.

#include "decode_internal.h"
#include "kvattn_kernel.h"

namespace tq {
namespace {

struct ScopePlan {
  bool plain, sinks;    // neither: shared
  Plan all, stack, rest;
  size_t parts, pre;    // bytes behind the counts
};

bool plan(const KvDev& c, const AttnCall& a, const ScopeCall& sc, ScopePlan* p) {
  const int share = a.n_heads / c.H;
  p->plain = p->sinks = false;
  if (sc.n_groups > 0 && a.window == 0) {
    const int64_t prefix = sc.max_prefix > 0 ? sc.max_prefix : length_hint(c, a);
    const int64_t tail = sc.max_tail > 0 ? (int64_t)sc.max_tail + 31 : length_hint(c, a);
    if (plan(c, (int64_t)a.n_tokens * share, sc.n_groups, prefix, &p->stack) &&
        plan(c, (int64_t)a.max_q * share, a.n_rows, tail, &p->rest)) {
      const size_t x = part_bytes(c, p->stack), y = part_bytes(c, p->rest);
      p->parts = x > y ? x : y;
      p->pre = (size_t)a.n_tokens * a.n_heads * (c.D + 4) * 4;
      return true;
    }
  }
  p->sinks = a.window > 0 && sc.sinks > 0;
  p->plain = !p->sinks;
  if (p->plain) return true;
  int64_t len = length_hint(c, a);
  const int64_t most = (int64_t)a.window + a.max_q + sc.sinks + 31;
  if (len > most) len = most;
  return plan(c, (int64_t)a.max_q * share, a.n_rows, len, &p->all);
}

// The leading pages that the rows of a group name alike.  A workgroup takes a
// group, 256 pages at a time; the first one also the rows that no group has.
__global__ void __launch_bounds__(256) shared_prefix_kernel(KvDev c, const int32_t* __restrict__ seqs,
                                                            const int32_t* __restrict__ cu, int n_groups, int n_rows,
                                                            int32_t* __restrict__ prefix) {
  __shared__ int lead, count, least, first;
  const int g = blockIdx.x, tid = threadIdx.x;
  const int64_t room = (int64_t)c.max_pages << c.page_shift;
  auto slot_of = [&](int r) {
    const int s = seqs ? seqs[r] : r;
    return s >= 0 && s < c.n_seqs && c.lens[s] > 0 ? s : -1;
  };
  if (g == 0 && cu != nullptr) {
    for (int r = tid; r < min(cu[0], n_rows); r += 256) prefix[r] = 0;
    for (int64_t r = (int64_t)max(cu[n_groups], 0) + tid; r < n_rows; r += 256) prefix[r] = 0;
  }
  const int r0 = cu ? cu[g] : 0, r1 = cu ? cu[g + 1] : n_rows;
  if (r0 < 0 || r1 > n_rows || r0 >= r1) return;
  if (tid == 0) {
    lead = first = INT32_MAX;
    count = 0;
    least = INT32_MAX;
  }
  __syncthreads();
  for (int r = r0 + tid; r < r1; r += 256) {
    const int s = slot_of(r);
    if (s < 0) continue;
    atomicMin(&lead, r);
    atomicAdd(&count, 1);
    atomicMin(&least, (int)min((int64_t)c.lens[s], room));
  }
  __syncthreads();
  // `first`: the first page that some row names otherwise or that is none.
  const int n = count > 1 ? (least + c.page_size - 1) >> c.page_shift : 0;
  const int32_t* mine = n > 0 ? c.pages + (int64_t)slot_of(lead) * c.max_pages : nullptr;
  for (int p0 = 0; p0 < n; p0 += 256) {
    const int p = p0 + tid;
    if (p < n) {
      const int page = mine[p];
      bool same = page >= 0 && page < c.n_pages;
      for (int r = lead + 1; r < r1; ++r) {
        const int s = slot_of(r);
        if (s >= 0) same &= c.pages[(int64_t)s * c.max_pages + p] == page;
      }
      if (!same) atomicMin(&first, p);
    }
    __syncthreads();
    if (first != INT32_MAX) break;
  }
  const int tokens = n > 0 ? (int)min((int64_t)min(first, n) << c.page_shift, (int64_t)least) : 0;
  for (int r = r0 + tid; r < r1; r += 256) prefix[r] = slot_of(r) >= 0 ? tokens : 0;
}

}  // namespace

bool kv_scope_plan(const KvDev& c, const AttnCall& a, const ScopeCall& sc, size_t* ws_bytes) {
  ScopePlan p;
  if (!plan(c, a, sc, &p)) return false;
  if (p.plain) return kv_attention_plan(c, a, ws_bytes);
  if (p.sinks)
    *ws_bytes = p.all.shares > 0 ? kCountBytes + part_bytes(c, p.all) : 0;
  else
    *ws_bytes = kCountBytes + p.parts + p.pre;
  return true;
}

hipError_t launch_kv_attention_scope(const KvDev& c, int layer, const AttnCall& call, const ScopeCall& sc,
                                     hipStream_t s) {
  ScopePlan p;
  if (!plan(c, call, sc, &p)) return hipErrorInvalidValue;
  if (p.plain) return launch_kv_attention(c, layer, call, s);
  MoreArgs a;
  a.cu_rows = sc.cu_rows;
  a.prefix = sc.prefix;
  a.pre = nullptr;
  a.pre_part = 0;
  a.pre_parts = 0;
  a.all_rows = call.n_rows;
  a.sinks = sc.sinks;
  if (p.sinks) {
    fill(a, c, layer, call, p.all);
    return start<kSinks>(c, a, p.all, s);
  }
  a.pre = reinterpret_cast<float*>(static_cast<uint8_t*>(call.ws) + kCountBytes + p.parts);
  a.pre_part = (int64_t)call.n_tokens * call.n_heads * (c.D + 4);
  a.pre_parts = 1;
  fill(a, c, layer, call, p.stack);
  a.n_rows = sc.n_groups;
  hipError_t e = start<kStack>(c, a, p.stack, s);
  if (e != hipSuccess) return e;
  fill(a, c, layer, call, p.rest);
  return start<kRest>(c, a, p.rest, s);
}

hipError_t launch_kv_shared_prefix(const KvDev& c, const int32_t* seqs, const int32_t* cu_rows, int n_groups,
                                   int n_rows, int32_t* prefix, hipStream_t s) {
  shared_prefix_kernel<<<n_groups, 256, 0, s>>>(c, seqs, cu_rows, n_groups, n_rows, prefix);
  return hipGetLastError();
}

}  // namespace tq
