// Attention over the 4-bit paged cache with sinks beside a window, and of
// rows that share the pages of a prefix (gfx950).
//
// Sinks: the records of a tile are those of its window and, in front of them,
// the first ones of the slot; masks in the records where they end.  The host
// decides the parts and the waves (8 of them to a tile where the chip is not full:
// 32 rows of 8 heads behind a window of 1024 and 4 sinks 15.3 us; the launch that
// rows without sinks still take needs 23.6 behind the same window).
//
// Shared prefixes.  The softmax over all tokens of a row is joined from those over
// any parts of them: with m the largest logit of a part, l = sum exp(s - m) and
// y = sum exp(s - m) v,
//     o = sum_parts exp(m - M) y / sum_parts exp(m - M) l,   M = max of the m.
// One launch takes the queries of all rows of a group as the rows of its tiles
// over the shared records, and every row over what it has behind them; a second
// one joins.  A query of a row that asks for more of them than it holds tokens may see
// none: its sums are 0 in every part then.  (Unpacking a record once into LDS for 128 or 256 stacked rows, as two
// fp16 halves of every value, took 1.3 to 1.8 times as long up to 8192 shared
// tokens, and as long with its additional launch at 64 rows x 32768.)
//
// What bounds it (8 heads of 128, groups of 64): 64 rows x 4 heads over 32768
// shared tokens 108 us, of which vector instructions, 391 a record and tile, are 85
// and matrix instructions 21; 16 rows over 8000 18: eight records a wave behind a
// chain of loads (16 heads of 256 on 4: 31 in groups of 64, 38 in groups of 32).  The
// join 4 to 6.  tq_kv_shared_prefix, a workgroup a group that walks its rows: 16 rows
// of 125 pages 6.4, 64 of 512 44, 512 of 32 in eight groups 20 and in one 113.

#include "decode_internal.h"
#include "kvattn_kernel.h"

namespace tq {
namespace {

struct ScopePlan {
  bool plain, sinks;    // neither: shared
  int waves;            // of a workgroup of kv_attn_kernel
  int tiles, parts;     // of a row, 16 query rows each; of its own tokens
  int stack_tiles, stack_parts;   // of all groups; of a group's shared tokens
  size_t bytes;         // workspace behind the counts
};

// Records of each of `ids` tiles and heads.
struct Work {
  int64_t ids, recs;
};

// What a launch of workgroups of `waves` waves takes (us), where `a` and `b` are cut
// into parts.  A CU has its share of the workgroups of `a`, a whole number, and of
// those of `b`.  A record takes a wave alone on its SIMD 1, two waves 1.6 and three 2.3;
// 2.5 start and end a round of workgroups of four waves, 3.5 of eight; 0.12 joins a part.  (64 rows of 4 heads over
// 32768 shared tokens, of which 128 tiles and heads are cut into 1, 2, 3, 4, 6, 8 parts:
// 264, 140, 150, 117, 113, 113 us; 16 rows over 8000, 32 of them into 5, 6, 7, 8, 10, 12,
// 15, 18: 24.8, 22.9, 21.1, 20.3, 23.6, 22.2, 20.9, 22.8.)
double cost(const KvDev& c, int waves, Work a, int parts_a, Work b, int parts_b) {
  const int lds = waves * 16 * (c.D + 6) * 4, by_lds = 160 * 1024 / lds, by_waves = 4 * waves_of(c.D, c.G) / waves;
  const int64_t slots = (int64_t)kCus * (by_lds < by_waves ? by_lds : by_waves);
  const int64_t n_a = a.ids * parts_a, n_b = b.ids * parts_b, rounds = (n_a + n_b + slots - 1) / slots;
  const double recs_a = a.ids > 0 ? (double)((a.recs + parts_a * waves - 1) / (parts_a * waves)) : 0.0;
  const double recs_b = b.ids > 0 ? (double)((b.recs + parts_b * waves - 1) / (parts_b * waves)) : 0.0;
  const double longest = recs_a > recs_b ? recs_a : recs_b;
  const double of_simd = (double)((n_a + kCus - 1) / kCus) * a.recs / (4.0 * parts_a) + (double)b.ids * b.recs / (4.0 * kCus);
  const double busy = 0.73 * of_simd + 0.13 * longest;
  return (waves == 8 ? 3.5 : 2.5) * rounds + (busy > longest ? busy : longest) + 0.12 * (parts_a + parts_b);
}

// The best parts of `a` beside `b`, in workgroups of `waves` waves; `join`: what
// another launch that joins parts takes.  A part is a record a wave at least, and all
// of them fit a grid, which holds fewer than 2^32 threads (1e30 where none do).
double split(const KvDev& c, int waves, Work a, Work b, int parts_b, double join, int* parts) {
  double best = 1e30;
  for (int n = 1; n <= kMaxParts && (n == 1 || a.recs >= (int64_t)waves * n); n += n < 16 ? 1 : n / 8) {
    if ((a.ids * n + b.ids * parts_b) * waves * 64 >= (int64_t)1 << 32) break;
    const double t = cost(c, waves, a, n, b, parts_b) + (n > 1 ? join : 0.0);
    if (t < best) {
      best = t;
      *parts = n;
    }
  }
  return best;
}

bool plan(const KvDev& c, const AttnCall& a, const ScopeCall& sc, ScopePlan* p) {
  const int share = a.n_heads / c.H;
  const int64_t rows = (int64_t)a.max_q * share, tiles = (rows + 15) / 16, ids = tiles * a.n_rows * c.H;
  const int64_t hint = length_hint(c, a), part_bytes = (int64_t)a.n_tokens * a.n_heads * (c.D + 4) * 4;
  // What a grid holds in one part: with 256 threads a workgroup, and with 512 of two kinds.
  constexpr int64_t kMostIds = 1 << 23, kMostOfTwo = 1 << 21;
  p->plain = p->sinks = false;
  p->stack_parts = p->stack_tiles = 0;
  p->waves = 4;
  p->tiles = (int)tiles;
  p->bytes = 0;
  if (tiles > 65535 || ids > kMostIds) return false;
  if (sc.n_groups > 0 && a.window == 0 && a.n_tokens < 1 << 24) {   // (what a grid of tokens holds)
    const int64_t stacked = (int64_t)a.n_tokens * share;
    const int64_t prefix = (sc.max_prefix > 0 ? sc.max_prefix : hint) / 32;
    const int64_t tail = (sc.max_tail > 0 ? (int64_t)sc.max_tail + 31 : hint) / 32 + 1;
    const int64_t stack_tiles = (stacked + 15) / 16 + sc.n_groups - 1, stack_ids = stack_tiles * c.H;
    if (ids <= kMostOfTwo && stack_ids <= kMostOfTwo) {
      p->stack_tiles = (int)stack_tiles;
      const Work stack{stack_ids, prefix}, rest{ids, tail}, none{0, 0};
      split(c, 4, rest, none, 1, 0.0, &p->parts);
      double t = split(c, 4, stack, rest, p->parts, 0.0, &p->stack_parts);
      p->waves = 4;
      if (c.D != 256) {
        int n;
        const double t8 = split(c, 8, stack, rest, p->parts, 0.0, &n);
        if (t8 < t) {
          t = t8;
          p->waves = 8;
          p->stack_parts = n;
        }
      }
      int n;
      const double alone = split(c, 4, Work{ids, prefix + tail}, none, 1, 8.0, &n);
      t += 6.0;   // the second launch
      if (t < alone) {
        p->bytes = (size_t)(p->parts + p->stack_parts) * part_bytes;
        return true;
      }
    }
  }
  p->stack_parts = 0;
  p->sinks = a.window > 0 && sc.sinks > 0;
  p->plain = !p->sinks;
  if (p->plain) return true;
  const int64_t most = (int64_t)a.window + a.max_q + sc.sinks + 31, len = hint < most ? hint : most;
  const Work all{ids, len / 32 + 1}, none{0, 0};
  int n;
  p->waves = 4;
  const double t = split(c, 4, all, none, 1, 6.0, &p->parts);
  if (c.D != 256 && ids <= kMostOfTwo && split(c, 8, all, none, 1, 6.0, &n) < t) {
    p->waves = 8;
    p->parts = n;
  }
  if (a.max_q > 65535) p->parts = 1;   // a grid of rows and tokens
  if (p->parts > 1) p->bytes = (size_t)p->parts * part_bytes;
  return true;
}

template <int MODE>
hipError_t start(const KvDev& c, const MoreArgs& a, const ScopePlan& p, hipStream_t s) {
  const dim3 grid(a.stack_blocks + a.H * a.parts * a.n_rows * a.tiles);
  return with_sizes(c, [&](auto D, auto G) {
    if constexpr (D() != 256)
      if (p.waves == 8) {
        kv_attn_kernel<D(), G(), MODE, 8><<<grid, 64 * 8, 0, s>>>(a);
        return;
      }
    kv_attn_kernel<D(), G(), MODE, 4><<<grid, 64 * 4, 0, s>>>(a);
  });
}

template <int MODE>
hipError_t start_join(const KvDev& c, const MoreArgs& a, hipStream_t s) {
  const dim3 grid = MODE == kShared ? dim3(a.n_tokens, a.H * a.share) : dim3(a.H * a.share, a.n_rows, a.max_q);
  if (c.D == 64)
    kv_join_kernel<64, MODE><<<grid, 256, 0, s>>>(a);
  else if (c.D == 128)
    kv_join_kernel<128, MODE><<<grid, 256, 0, s>>>(a);
  else
    kv_join_kernel<256, MODE><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
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
    const int found = first;
    __syncthreads();   // all have looked before the next pages can change it
    if (found != INT32_MAX) break;
  }
  const int tokens = n > 0 ? (int)min((int64_t)min(first, n) << c.page_shift, (int64_t)least) : 0;
  for (int r = r0 + tid; r < r1; r += 256) prefix[r] = slot_of(r) >= 0 ? tokens : 0;
}

}  // namespace

bool kv_scope_plan(const KvDev& c, const AttnCall& a, const ScopeCall& sc, size_t* ws_bytes) {
  ScopePlan p;
  if (!plan(c, a, sc, &p)) return false;
  if (p.plain) return kv_attention_plan(c, a, ws_bytes);
  *ws_bytes = p.bytes > 0 ? kCountBytes + p.bytes : 0;
  return true;
}

hipError_t launch_kv_attention_scope(const KvDev& c, int layer, const AttnCall& call, const ScopeCall& sc,
                                     hipStream_t s) {
  ScopePlan p;
  if (!plan(c, call, sc, &p)) return hipErrorInvalidValue;
  if (p.plain) return launch_kv_attention(c, layer, call, s);
  MoreArgs a;
  fill(a, c, layer, call, Plan{p.tiles, 0, 0, 0});
  a.cu_rows = sc.cu_rows;
  a.prefix = sc.prefix;
  a.pre = a.part;   // behind the counts, which are not used
  a.pre_part = (int64_t)call.n_tokens * call.n_heads * (c.D + 4);
  a.parts = p.parts;
  a.stack_parts = p.stack_parts;
  a.n_groups = sc.n_groups;
  a.stack_blocks = 0;
  a.sinks = sc.sinks;
  hipError_t e;
  if (p.sinks) {
    e = start<kSinks>(c, a, p, s);
    return e == hipSuccess && p.parts > 1 ? start_join<kSinks>(c, a, s) : e;
  }
  a.stack_blocks = c.H * p.stack_parts * p.stack_tiles;
  e = start<kShared>(c, a, p, s);
  return e == hipSuccess ? start_join<kShared>(c, a, s) : e;
}

hipError_t launch_kv_shared_prefix(const KvDev& c, const int32_t* seqs, const int32_t* cu_rows, int n_groups,
                                   int n_rows, int32_t* prefix, hipStream_t s) {
  shared_prefix_kernel<<<n_groups, 256, 0, s>>>(c, seqs, cu_rows, n_groups, n_rows, prefix);
  return hipGetLastError();
}

}  // namespace tq
