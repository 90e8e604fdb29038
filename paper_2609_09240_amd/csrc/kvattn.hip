// Attention over the 4-bit paged cache (gfx950), one pass over the keys and
// values with the running maximum and sum of the softmax:
//     s_j = scale * sum_g ( sk_jg ((q . ck_j)_g + 8 sum_g q) + mk_jg sum_g q )
//     o   = sum_j ( p_j sv_jg ) cv_j  +  sum_j p_j (mv_jg + 8 sv_jg),   p_j = exp(s_j - max) / sum
// ck, cv: the codes less 8; sk, mk, sv, mv: scale and offset of token j's group
// g of channels.  No key or value is formed: the codes are exact
// operands of the matrix instructions and the parameters multiply the fp32
// sums (keys) or the probabilities (values).
//
// One wave takes records of 32 tokens against a tile of 16 query rows (a
// row is a query token and one of the heads that share the key/value head):
//   S^T = K Q^T: 16 tokens x 16 rows per instruction, a lane's four sums are
//   four tokens of the row lane % 16, and the eight it holds of a record are
//   its operand of the second product as they stand, since values are stored
//   with those eight tokens in one word: O^T += V^T P^T.
// A probability times a value scale enters as two fp16 numbers (hi + lo, 22
// bits), in a unit of the row and group that follows the largest scale seen;
// the sums of p, of p (mv + 8 sv) and of everything else are fp32.
//
// Work split: a workgroup has four waves that take the records of its range
// in turn and join their references, sums and outputs through LDS.  Where there
// are few tiles over long caches the records of all of them are laid in a
// line and divided evenly among as many workgroups as the chip holds, whatever
// the lengths are; a tile that several workgroups have parts of is joined by
// the last of them to finish.  Otherwise a workgroup has a tile: also where there
// are more than 256 tiles and rows, one of them over a long cache or not (300
// rows, one of them 131072 tokens long: 1036 us; 200: 69).
//
// A record's 4.6 KB (D = 128, groups of 64) arrive in the registers of the
// record before, each as soon as it is used; 168 of them allow three waves a
// SIMD.  One token over one long cache: 5.4 TB/s for every further byte, and
// 6 us of launch, table, first loads and joining waves before the first, 7 us
// for joining 96 parts a head.
//   1 x 131072 tokens, 8 heads, groups of 128 (143 MB)  40.2 us
//   32 ragged rows to 8192, groups of 64 (93 MB)        34.3
//   1 x 4096 (4.7 MB)                                   12.0
//   1 x 45                                              6.4
//   8 x 8 queries of ragged rows to 8192 (31 MB)        34.6
//   a chunk of 2 x 1000 queries over up to 5000, window 2048, 14 heads of 64 on
//   2, groups of 32 (10 GFLOP)                          82
// A unit a group cost 1 to 5 % of these (the largest scale of a record, and a
// multiplication a probability and group behind the first).
// (One launch a split and another to join: 31 + 6.5, 33 + 6 and 10 + 6 for the
// first three, and 3 us between the launches.  32 or 64 rows a tile, which
// unpack a record once for two or four tiles, halve the waves: 90 and 120 us
// where the chunk took 77, 37 where 8 queries of 4 heads took 29.)

#include "q4_internal.h"

namespace tq {
namespace {

constexpr int kWaves = 4;

// The page table as memory that no launch in flight writes: uniform reads of
// it are scalar loads.
typedef const __attribute__((address_space(4))) int32_t* table_ptr;
__device__ inline table_ptr as_table(const int32_t* p) { return (table_ptr)(uintptr_t)p; }
constexpr int kCus = 256;
// Up to kMinUnits units (512 tokens) a tile is one workgroup's: a second one
// saves less than joining costs.  A share has kUnitsOfShare units at least
// (4096 tokens: 13.9 us with one, 12.2 with two, 13.7 with four).
constexpr int kMinUnits = 4;
constexpr int kUnitsOfShare = 2;
constexpr int kMaxShares = 4 * kCus;
constexpr int kOneLevel = 16;   // parts joined in one step (96 of them: 47 us in one step, 40 in two)
constexpr float kLn2 = 0.69314718055994531f;

__device__ inline float4v mfma(half8 a, half8 b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// What a probability times a value scale is held in.  The running reference
// of a row (log2) is kept so that its largest probability so far lies in 2^12 ..
// 2^14, and a unit of each group, a power of two, so that the largest scale seen
// lies in 1 .. 2 units: the product is below 2^15, which fp16 takes, and what
// two halves leave out is 2^-21 of it or, rounded, 2^-25, which is 2^-37 of the
// largest probability times the largest scale.  (One unit for all groups would
// cost an ordinary group the bits that an outlier in another one needs, and a
// fixed one those of small scales.)  The reference holds the unit of group 0 as
// well, whose products need no multiplication for it then.
constexpr float kHigh = 14.0f, kHighSet = 12.0f;

__device__ inline half2v pair(uint32_t b) { return __builtin_bit_cast(half2v, b); }

// The pair with the largest scale, in its low half; as whole numbers, which have
// the order of the scales (NaN is the largest).  The upper half may be anything.
__device__ inline uint32_t larger(uint32_t a, uint32_t b) {
  typedef uint16_t us2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, a), __builtin_bit_cast(us2, b)));
}
// Of three at a time, four instructions for eight in place of seven, which heads
// of 256 have no registers for.
template <int D>
__device__ inline uint32_t largest(uint32_t a, uint32_t b, uint32_t c) {
  if constexpr (D == 256) return larger(larger(a, b), c);
  uint32_t d;
  asm("v_max3_u16 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
  return d;
}

// f over the four lanes that hold a row's tokens (16 lanes apart), in each of them.
template <class F>
__device__ inline uint32_t over_row(uint32_t x, F f) {
  const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = f(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return f(b[0], b[1]);
}

// Two fp32 numbers as fp16 rounded towards 0, and what that left.
__device__ inline uint32_t cut(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(a, b));
}
__device__ inline float rest0(uint32_t h, float w) {
  float d;
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(d) : "v"(h), "v"(w));
  return d;
}
__device__ inline float rest1(uint32_t h, float w) {
  float d;
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(d) : "v"(h), "v"(w));
  return d;
}

// For x in 2^e .. 2^(e + 1): 2^e, 2^-e and e.
__device__ inline float power_of(float x) { return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x) & 0x7F800000u); }
__device__ inline float over_power(float x) {
  return __builtin_bit_cast(float, 0x7F000000u - (__builtin_bit_cast(uint32_t, x) & 0x7F800000u));
}
__device__ inline float log2_of(float x) { return (float)((int)(__builtin_bit_cast(uint32_t, x) >> 23) - 127); }

struct Args {
  const uint8_t* layer;    // the layer's pages
  const int32_t* pages;
  const int32_t* lens;
  const int32_t* seqs;
  const int32_t* cu;
  const uint16_t* q;
  void* o;
  float* lse;
  int32_t* count;          // [2][2 * kMaxShares] parts and groups of parts that have arrived, 0 between calls
  float* part;             // [2 * workgroups][R][D + 4]: sums, reference (log2), sum of p
  int64_t q_ts, q_hs, page_bytes;
  float scale_log2;
  int32_t n_rows, n_tokens, max_q, H, share, window;
  uint32_t share_magic;    // floor(2^32 / share) + 1
  int32_t page_shift, n_seqs, max_pages, n_pages;
  int32_t tiles;           // tiles of a row
  int32_t shares;          // workgroups that divide the work evenly; 0: one per tile and head
  int32_t R;               // rows of a tile kept in the workspace
  int32_t out_f32;
};

// What a tile of rows is: row b of the call, key/value head h, tile qt.
struct Tile {
  int b, h, qt;
  int seq, first, n, rows;   // slot, first token in q, tokens, rows of (b, h) in all
  int64_t asked;             // tokens the call names for the row, max_q or not
  int len;
  int row0, tok0, head0;     // first of the tile's rows, its token and head
  int rec0, rec1;            // records it can see
  int units;                 // of four records, one a wave; 1 where there are none
};

// x / share for x < share + 16 <= 2^16.
__device__ inline int by_share(const Args& a, int x) {
  return a.share == 1 ? x : (int)__umulhi((uint32_t)x, a.share_magic);
}

// Tile (b, qt) of head 0; false where there is none.
__device__ inline bool tile_of(const Args& a, int b, int qt, Tile* t) {
  t->h = 0;
  t->b = b;
  t->qt = qt;
  t->seq = a.seqs ? as_table(a.seqs)[b] : b;
  int64_t first = a.cu ? as_table(a.cu)[b] : b, end = a.cu ? as_table(a.cu)[b + 1] : (int64_t)b + 1;
  const int64_t asked = t->asked = end - first;
  const bool bad = first < 0 || asked < 0;
  end = min(min(end, (int64_t)a.n_tokens), first + a.max_q);
  t->first = (int)first;
  t->n = bad || end <= first ? 0 : (int)(end - first);
  t->rows = t->n * a.share;
  t->row0 = qt * 16;
  if (t->row0 >= t->rows) return false;
  t->tok0 = qt == 0 ? 0 : t->row0 / a.share;
  t->head0 = t->row0 - t->tok0 * a.share;
  t->len = 0;
  if (t->seq >= 0 && t->seq < a.n_seqs)
    t->len = (int)min(min(max((int64_t)as_table(a.lens)[t->seq], (int64_t)0), (int64_t)a.max_pages << a.page_shift),
                      (int64_t)INT32_MAX - 64);
  // Position of query token i is base + i; all of what was asked for counts.
  const int64_t base = t->len - asked;
  const int last = min(t->tok0 + by_share(a, t->head0 + 15), t->n - 1);
  const int64_t hi = min((int64_t)t->len, base + last + 1);
  const int64_t lo = a.window > 0 ? max((int64_t)0, base + t->tok0 + 1 - a.window) : 0;
  t->rec0 = (int)(lo >> 5);
  t->rec1 = hi > lo ? (int)((hi + 31) >> 5) : t->rec0;
  t->units = max(1, (t->rec1 - t->rec0 + kWaves - 1) / kWaves);
  return true;
}

// o and lse of row r of a tile: four channels of the joined sum y, what it is
// divided by, the reference.
__device__ inline void store_row(const Args& a, const Tile& t, int D, int r, int d, float4v y, float sum, float ref) {
  const int tok = by_share(a, t.head0 + r), head = t.head0 + r - tok * a.share;
  const int64_t at = (int64_t)(t.first + t.tok0 + tok) * (a.H * a.share) + t.h * a.share + head;
  y *= sum == 0.0f ? 0.0f : 1.0f / sum;
  if (a.out_f32) {
    *reinterpret_cast<float4v*>(static_cast<float*>(a.o) + at * D + d) = y;
  } else {
    const half4 z = {(_Float16)y[0], (_Float16)y[1], (_Float16)y[2], (_Float16)y[3]};
    *reinterpret_cast<half4*>(static_cast<uint16_t*>(a.o) + at * D + d) = z;
  }
  if (a.lse && d == 0) a.lse[at] = sum == 0.0f ? -__builtin_inff() : (ref + log2f(sum)) * kLn2;
}

// Even shares: the units of all tiles and heads in a line (tiles by qt, then
// row, then head), which W workgroups divide: the first T % W take one more than
// the others.  A pair is a tile and row, qt * n_rows + row; up to 256 of them, up
// to four beside each other in a lane.
constexpr int kMaxPairs = 256;

// A workgroup's share: units [unit, end) of T, the first of them unit `off` of
// pair `pair`.  Every wave works it out for itself.
struct Share {
  int q, more;             // units of every share, and how many shares have one more
  int unit, end, pair, off;
};
__device__ inline int share_start(const Share& s, int w) { return w * s.q + min(w, s.more); }
__device__ inline int share_with(const Share& s, int unit) {
  const int head = s.more * (s.q + 1);
  return unit < head ? unit / (s.q + 1) : s.more + (unit - head) / s.q;
}
__device__ inline Share share_of(const Args& a) {
  const int lane = threadIdx.x & 63, pairs = a.n_rows * a.tiles, per = (pairs + 63) >> 6;
  int n[kMaxPairs / 64], sum = 0;
#pragma unroll
  for (int e = 0; e < kMaxPairs / 64; ++e) {
    const int i = lane * per + e;
    n[e] = 0;
    if (e < per && i < pairs) {
      Tile t;
      const int qt = a.tiles == 1 ? 0 : i / a.n_rows;
      if (tile_of(a, i - qt * a.n_rows, qt, &t)) n[e] = t.units * a.H;
    }
    sum += n[e];
  }
  const int incl = wave_scan(sum);
  Share s;
  const int T = __builtin_amdgcn_readlane(incl, 63), W = min(a.shares, T);
  s.q = s.more = s.unit = s.end = s.pair = s.off = 0;
  if ((int)blockIdx.x >= W) return s;
  s.q = T / W;
  s.more = T - s.q * W;
  s.unit = share_start(s, blockIdx.x);
  s.end = share_start(s, blockIdx.x + 1);
  // The last lane, then pair, that starts at or before the unit.
  const int at = __popcll(__builtin_amdgcn_ballot_w64(incl - sum <= s.unit)) - 1;
  s.pair = at * per;
  s.off = s.unit - __builtin_amdgcn_readlane(incl - sum, at);
#pragma unroll
  for (int e = 0; e < kMaxPairs / 64 - 1; ++e) {
    const int here = __builtin_amdgcn_readlane(n[e], at);
    if (s.pair == at * per + e && s.off >= here) {
      s.off -= here;
      ++s.pair;
    }
  }
  return s;
}

// Everything of a record that a lane needs, as it lies in memory.
template <int D, int G>
struct Record {
  uint32_t k[2][D / 32];
  u4v v[D / 64];
  u4v kp[D / G][2], vp[D / G][2];
};

// The kernel's arguments read anew: what a stretch of code needs of them holds
// no scalar registers outside of it.  (41 to 52 of those live in lanes of vector
// registers meanwhile; with all arguments kept, 111 to 127, and some variants
// spill vector registers for them.)
__device__ inline Args args_anew() {
  typedef const __attribute__((address_space(4))) Args* ptr;
  ptr p = (ptr)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const Args*)p;
}

// Waves a SIMD holds of a variant, as many as its vector registers allow without
// a spill (512 / waves of them; past 256 half of them are accumulation registers
// that cost moves).
constexpr int waves_of(int D, int G) { return D == 64 ? 4 : D == 128 ? (G == 32 ? 2 : 3) : 1; }

template <int D, int G>
__global__ void __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(waves_of(D, G))))
kv_attn_kernel(Args args) {
  constexpr int NG = D / G, J = G / 32, KD = D / 32, VD = D / 16;
  constexpr int64_t kRec = 32 * (D + 8 * NG);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane >> 4;
  __shared__ float sm[kWaves][16], sl[kWaves][16];
  __shared__ float so[kWaves][16][D + 4];
  __shared__ int arrived;
  Share share = {1, 0, 0, 1, 0, 0};
  if (args.shares > 0) share = share_of(args);
  const int first_unit = share.unit;
  Tile t;
  int h = 0;
  bool fresh = true;   // the pair's tile is to be looked up
  // The tiles, or parts of tiles, of the workgroup: one, or those of its share.
  while (share.unit < share.end) {
  const Args a = args_anew();
  int rec0, rec1, head_unit = 0;
  bool all_of_it = true;
  const int slot = 2 * blockIdx.x + (share.unit != first_unit);
  if (a.shares > 0) {
    if (fresh) {
      for (;; ++share.pair) {   // there is one: units are left
        const int qt = a.tiles == 1 ? 0 : share.pair / a.n_rows;
        if (tile_of(a, share.pair - qt * a.n_rows, qt, &t)) break;
      }
      h = share.off / t.units;
      share.off -= h * t.units;
    }
    const int k0 = share.off, k1 = min(t.units, k0 + share.end - share.unit);
    head_unit = share.unit - k0;
    all_of_it = k0 == 0 && k1 == t.units;
    rec0 = t.rec0 + kWaves * k0;
    rec1 = min(t.rec1, t.rec0 + kWaves * k1);
    share.unit += k1 - k0;
    share.off = 0;
    t.h = h;
    fresh = ++h == a.H;
    if (fresh) ++share.pair;
  } else {
    if (!tile_of(a, blockIdx.y, blockIdx.z, &t)) return;
    t.h = blockIdx.x;
    rec0 = t.rec0;
    rec1 = t.rec1;
    share.unit = share.end;
  }

  // The same in every lane: scalar registers, whatever they were computed in.
  auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  rec0 = uniform(rec0);
  rec1 = uniform(rec1);
  t.rows = uniform(t.rows);
  t.row0 = uniform(t.row0);
  t.tok0 = uniform(t.tok0);
  t.head0 = uniform(t.head0);
  t.first = uniform(t.first);
  t.n = uniform(t.n);
  t.len = uniform(t.len);

  // The next record of the wave from `rec` on whose page the table names, as
  // the address of its bytes; null where there is none.
  const int per_shift = a.page_shift - 5;
  const table_ptr row_pages = as_table(a.pages) + (int64_t)(t.len > 0 ? t.seq : 0) * a.max_pages;
  auto next_record = [&](int* rec) -> const uint8_t* {
    for (; *rec < rec1; *rec += kWaves) {
      const int page = row_pages[*rec >> per_shift];
      if (page >= 0 && page < a.n_pages) {
        const int per = 1 << per_shift;
        return a.layer + (int64_t)page * a.page_bytes + ((int64_t)t.h * per + (*rec & (per - 1))) * kRec;
      }
    }
    return nullptr;
  };
  auto load_k = [&](Record<D, G>& r, const uint8_t* p) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint8_t* kp = p + (64 * h + lane) * (D / 8);
      if constexpr (D == 64) {
        const u2v x = *reinterpret_cast<const u2v*>(kp);
        r.k[h][0] = x[0];
        r.k[h][1] = x[1];
      } else {
#pragma unroll
        for (int i = 0; i < D / 128; ++i) {
          const u4v x = *reinterpret_cast<const u4v*>(kp + 16 * i);
#pragma unroll
          for (int e = 0; e < 4; ++e) r.k[h][4 * i + e] = x[e];
        }
      }
    }
  };
  auto load_v = [&](Record<D, G>& r, const uint8_t* p) {
#pragma unroll
    for (int i = 0; i < D / 64; ++i) r.v[i] = *reinterpret_cast<const u4v*>(p + 16 * D + (64 * i + lane) * 16);
  };
  // The parameters of tokens 4c .. 4c + 3 and 16 more of the keys (first 0) or
  // the values (first NG).
  auto load_params = [&](u4v (&x)[NG][2], const uint8_t* p, int first) {
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        x[g][h] = *reinterpret_cast<const u4v*>(p + 32 * D + (first + g) * 128 + (16 * h + 4 * c) * 4);
  };

  // The first record is on its way while the queries are set up.
  Record<D, G> r;
  int rec = rec0 + wave;
  const uint8_t* at = next_record(&rec);
  if (at != nullptr) {
    load_k(r, at);
    load_params(r.kp, at, 0);
    load_params(r.vp, at, NG);
    load_v(r, at);
  }

  // The lane's query rows as operands, their sums per group (and 8 times
  // them, what codes less 8 lack) in the codes' unit, their positions.
  int qx = threadIdx.x;
  asm volatile("" : "+v"(qx));   // as above the join, below
  const int qc = (qx >> 4) & 3, qcol = qx & 15;
  half8 q[KD];
  float qs[NG];
  float4v q8[NG];
  int pos;
  const int64_t base = (int64_t)t.len - t.asked;
  const half8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
  const bool in = t.row0 + qcol < t.rows;
  const int up = by_share(a, t.head0 + qcol), tok = in ? t.tok0 + up : 0;
  const int head = in ? t.h * a.share + t.head0 + qcol - up * a.share : 0;
  const uint16_t* qp = a.q + (int64_t)(t.first + tok) * a.q_ts + head * a.q_hs;
  pos = in ? (int)max(base + tok, (int64_t)-1) : -1;
#pragma unroll
  for (int j = 0; j < KD; ++j) q[j] = in ? load8(qp + 32 * j + 8 * qc) : zero;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += (float)q[g * J + j][e];
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    qs[g] = s / kCodeUnit;
    const float s8 = 8.0f / kCodeUnit * s;
    q8[g] = float4v{s8, s8, s8, s8};
  }
  // The positions between which every row of the tile sees every token.
  int all0 = 0, all1;
  {
    const int last = min(t.tok0 + by_share(a, t.head0 + 15), t.n - 1);
    all1 = (int)max((int64_t)0, min((int64_t)t.len, base + t.tok0 + 1));
    if (a.window > 0) all0 = (int)max((int64_t)0, base + last + 1 - a.window);
    all0 = uniform(all0);
    all1 = uniform(all1);
  }

  const float logit = a.scale_log2 * kCodeUnit;

  // A row's state: its reference r, above which a logit makes it grow (never
  // before it has seen one: then any does), sums of exp2(s - r).
  const float kNone = -3.0e38f;
  float4v acc[VD];
  float macc[NG], ref, grow, l;
  // Twice the unit of group 0 (a power of two that ref holds: its logarithm is
  // added), and that unit over the other groups'.  At first the smallest scale
  // there is.
  float unit2 = 0x1p-23f, per_unit[NG];
  ref = 0.0f;
  grow = kNone;
  l = 0.0f;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    macc[g] = 0.0f;
    per_unit[g] = 1.0f;
  }
#pragma unroll
  for (int j = 0; j < VD; ++j) acc[j] = float4v{0, 0, 0, 0};
  // Some row of the wave has sums that are not 0 (or are NaN): what its first
  // record brings has nothing to rescale.  (Heads of 256 would spill.)
  auto begun = [&] { return D == 256 || __builtin_amdgcn_ballot_w64(l != 0.0f) != 0; };
  auto rescale = [&](float f) {
    l *= f;
#pragma unroll
    for (int g = 0; g < NG; ++g) macc[g] *= f;
#pragma unroll
    for (int j = 0; j < VD; ++j) acc[j] *= f;
  };

  while (at != nullptr) {
    // A register's record is replaced by the next one's as soon as it is used,
    // so that a load has nearly a whole pass to arrive in.
    int rec_n = rec + kWaves;
    const uint8_t* at_n = next_record(&rec_n);
    const uint8_t* pf = at_n != nullptr ? at_n : at;
    const bool whole = rec * 32 >= all0 && rec * 32 + 32 <= all1;
    half8 kf[2][KD];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < KD; ++j) kf[h][j] = code_operand(r.k[h][j]);
    u4v hi[NG], lo[NG];
    float s[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float x[4] = {0, 0, 0, 0};
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        float4v z = q8[g];
#pragma unroll
        for (int j = 0; j < J; ++j) z = mfma(kf[h][g * J + j], q[g * J + j], z);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const half2v p = pair(r.kp[g][h][i]);
          x[i] = fmaf((float)p[0], z[i], x[i]);
          x[i] = fmaf((float)p[1], qs[g], x[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) s[h][i] = fmaf(x[i], logit, -ref);
    }
    load_k(r, pf);
    u4v vp[NG][2];
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int h = 0; h < 2; ++h) vp[g][h] = r.vp[g][h];
    if (!whole) {
      asm volatile("");   // a branch: as selects the masks cost every record 40 instructions
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int tok = rec * 32 + 16 * h + 4 * c + i;
          const bool see = tok <= pos && (a.window <= 0 || tok > pos - a.window);
          if (!see) s[h][i] = -__builtin_inff();
#pragma unroll
          for (int g = 0; g < NG; ++g) vp[g][h][i] = see ? vp[g][h][i] : 0u;   // may be anything
        }
    }
    float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                      fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
    if (__builtin_amdgcn_ballot_w64(top > grow) != 0) {
      top = __builtin_bit_cast(float, over_row(__builtin_bit_cast(uint32_t, top), [](uint32_t a, uint32_t b) {
        return __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)));
      }));
      const bool some = begun();
      if (top > grow) {
        const float set = kHighSet - log2_of(0.5f * unit2), by = top - set;
        if (some) rescale(grow == kNone ? 0.0f : exp2f(-by));
        ref += by;
        grow = set + (kHigh - kHighSet);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[h][i] -= by;
      }
    }
    // The largest scale of a group among the tokens that the row sees.  (NaN, as
    // a number the largest there is, makes no unit larger.)
    uint32_t most[NG];
    float big = 0.0f;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const u4v x = vp[g][0], y = vp[g][1];
      most[g] = larger(largest<D>(largest<D>(x[0], x[1], x[2]), x[3], y[0]), largest<D>(y[1], y[2], y[3]));
      big = fmaxf(big, fmaf(lo_half(most[g]), per_unit[g], 0.0f));
    }
    if (__builtin_amdgcn_ballot_w64(big >= unit2) != 0) {
      const float unit0 = 0.5f * unit2;
      const bool some = begun();
      float now0 = unit0;
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const uint32_t x = over_row(most[g], larger);
        const float unit = unit0 * over_power(per_unit[g]), scale = lo_half(x);
        const float now = scale >= 2.0f * unit ? power_of(scale) : unit;
        if (g == 0) now0 = now;
        per_unit[g] = now0 * over_power(now);
        const float f = unit * over_power(now);
        if (some)
#pragma unroll
          for (int j = g * G / 16; j < (g + 1) * G / 16; ++j) acc[j] *= f;
      }
      // The reference and what is counted in it, for group 0.
      const float f = unit0 * over_power(now0), by = -log2_of(f);
      unit2 = 2.0f * now0;
      if (some) {
        l *= f;
#pragma unroll
        for (int g = 0; g < NG; ++g) macc[g] *= f;
      }
      ref += by;
      grow -= by;   // kNone stays what it is
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[h][i] -= by;
    }
    float p[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[h][i] = __builtin_amdgcn_exp2f(s[h][i]);
        l += p[h][i];
      }
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      // Operand register i: tokens 4c + i and 16 + 4c + i.
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const half2v v = pair(vp[g][h][i]);
          // One instruction with the fp16 operand as it is.  2^-25, half of what
          // the second half can hold, makes the cut to it a rounding.
          w[h] = fmaf(g == 0 ? p[h][i] : p[h][i] * per_unit[g], (float)v[0], 0x1p-25f);
          macc[g] = fmaf(p[h][i], fmaf(8.0f, (float)v[0], (float)v[1]), macc[g]);
        }
        const uint32_t x = cut(w[0], w[1]);
        hi[g][i] = x;
        lo[g][i] = cut(rest0(x, w[0]), rest1(x, w[1]));
      }
    }
    load_params(r.kp, pf, 0);
    load_params(r.vp, pf, NG);
#pragma unroll
    for (int j = 0; j < VD; ++j) {
      const half8 vf = code_operand(r.v[j >> 2][j & 3]);
      acc[j] = mfma(vf, __builtin_bit_cast(half8, hi[j * 16 / G]), acc[j]);
      acc[j] = mfma(vf, __builtin_bit_cast(half8, lo[j * 16 / G]), acc[j]);
    }
    load_v(r, pf);
    at = at_n;
    rec = rec_n;
  }

  // Join the four lane groups' sums, then the waves.  A row that has seen
  // nothing has the reference -infinity from here on.
  // (The thread's number is taken anew, so that what only this part needs of it
  // holds no registers meanwhile.)
  int tx = threadIdx.x;
  asm volatile("" : "+v"(tx));
  const Args z = args_anew();
  const __amdgpu_buffer_rsrc_t parts_of =
      __builtin_amdgcn_make_buffer_rsrc(z.part, 0, 2 * z.shares * z.R * (D + 4) * 4, 0x00020000);
  const int oc = (tx >> 4) & 3, ocol = tx & 15;
  const float m = grow == kNone ? -__builtin_inff() : ref;
  float L = l;
  L += __shfl_xor(L, 16);
  L += __shfl_xor(L, 32);
  float M[NG];
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    M[g] = macc[g] + __shfl_xor(macc[g], 16);
    M[g] += __shfl_xor(M[g], 32);
  }
  __syncthreads();   // what was joined before has been read
  if (oc == 0) sm[wave][ocol] = m;
  __syncthreads();
  float top = sm[0][ocol];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) top = fmaxf(top, sm[w][ocol]);
  const float f = m == -__builtin_inff() ? 0.0f : exp2f(m - top);
  if (oc == 0) sl[wave][ocol] = L * f;
#pragma unroll
  for (int j = 0; j < VD; ++j) {
    float4v y;
    const float unit = kCodeUnit / per_unit[j * 16 / G];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = fmaf(acc[j][i], unit, M[j * 16 / G]) * f;
    if (t.row0 + ocol < t.rows) *reinterpret_cast<float4v*>(&so[wave][ocol][16 * j + 4 * oc]) = y;
  }
  __syncthreads();
  for (int i = tx; i < 16 * D / 4; i += 64 * kWaves) {
    const int r = i / (D / 4), d = i % (D / 4) * 4, row = t.row0 + r;
    if (row >= t.rows) continue;
    float4v y = *reinterpret_cast<float4v*>(&so[0][r][d]);
    float sum = sl[0][r], most = sm[0][r];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
      y += *reinterpret_cast<float4v*>(&so[w][r][d]);
      sum += sl[w][r];
      most = fmaxf(most, sm[w][r]);
    }
    if (all_of_it) {
      store_row(z, t, D, r, d, y, sum, most);
    } else {
      const int p = (slot * z.R + r) * (D + 4) * 4;
      put4(parts_of, p + 4 * d, y);
      if (d == 0) put4(parts_of, p + 4 * D, float4v{most, sum, 0, 0});
    }
  }
  if (all_of_it) continue;

  // The last workgroup of a tile to leave its part joins them all, in the
  // order of the parts; where there are many, the last one of each group of
  // them joins the group into its first part, and the last group the groups.
  // Who finds a count full sets it back to 0.
  const int w0 = share_with(share, head_unit), parts = share_with(share, head_unit + t.units - 1) - w0 + 1;
  // Workgroup w0 comes to the tile after others unless its share starts there.
  const int skip = share_start(share, w0) != head_unit;
  auto slot_of = [&](int k) { return 2 * (w0 + k) + (k == 0 ? skip : 0); };
  const int g = parts > kOneLevel ? (int)ceilf(sqrtf((float)parts)) : parts, groups = (parts + g - 1) / g;
  int first = ((int)blockIdx.x - w0) / g * g, step = 1, n = min(g, parts - first);
  int32_t* count = z.count + slot_of(first);
  for (;;) {
  __builtin_amdgcn_s_waitcnt(0);   // what is joined has arrived
  __syncthreads();
  if (threadIdx.x == 0) {
    const int before = __hip_atomic_fetch_add(count, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (before == n - 1) __hip_atomic_store(count, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    arrived = before;
  }
  __syncthreads();
  if (arrived != n - 1) break;
  const bool last = step != 1 || groups == 1;
  asm volatile("" : "+v"(tx)::"memory");
  // D/4 lanes take a row, or each `per` of NGRP groups of them some of its parts.
  constexpr int kAhead = D == 64 ? 4 : 8;   // parts in flight a lane, as the registers allow
  constexpr int kLanes = D / 4, NGRP = 64 * kWaves / kLanes;
  const int rows = min(16, t.rows - t.row0), per = max(1, NGRP / rows);
  const int grp = tx / kLanes, d = tx % kLanes * 4;
  float(*jy)[D + 4] = so[0];   // NGRP <= 16 rows of it
  for (int r0 = 0; r0 < rows; r0 += NGRP / per) {
    const int r = r0 + grp / per, sub = grp % per;
    float ref = -__builtin_inff(), sum = 0.0f;
    float4v y = {0, 0, 0, 0};
    if (r < rows && grp < NGRP / per * per) {
      for (int s = sub; s < n; s += kAhead * per) {
        float4v v[kAhead];
        float m[kAhead], l[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
          const int k = first + step * min(s + e * per, n - 1);
          const int p = (slot_of(k) * z.R + r) * (D + 4) * 4;
          v[e] = get4(parts_of, p + 4 * d);
          const float4v x = get4(parts_of, p + 4 * D);
          m[e] = x[0];
          l[e] = x[1];
        }
        float top = ref;
#pragma unroll
        for (int e = 0; e < kAhead; ++e)
          if (s + e * per < n) top = fmaxf(top, m[e]);
        const float f = ref == -__builtin_inff() ? 0.0f : exp2f(ref - top);
        sum *= f;
        y *= f;
        ref = top;
#pragma unroll
        for (int e = 0; e < kAhead; ++e)
          if (s + e * per < n) {
            const float g = m[e] == -__builtin_inff() ? 0.0f : exp2f(m[e] - top);
            sum = fmaf(l[e], g, sum);
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = fmaf(v[e][i], g, y[i]);
          }
      }
    }
    __syncthreads();   // so has been read
    if (grp < NGRP) {
      *reinterpret_cast<float4v*>(&jy[grp][d]) = y;
      if (d == 0) {
        jy[grp][D] = ref;
        jy[grp][D + 1] = sum;
      }
    }
    __syncthreads();
    if (r < rows && sub == 0 && grp < NGRP / per * per) {
      float top = ref;
      for (int e = 1; e < per; ++e) top = fmaxf(top, jy[grp + e][D]);
      const float f = ref == -__builtin_inff() ? 0.0f : exp2f(ref - top);
      sum *= f;
      y *= f;
      for (int e = 1; e < per; ++e) {
        const float m = jy[grp + e][D], g = m == -__builtin_inff() ? 0.0f : exp2f(m - top);
        sum = fmaf(jy[grp + e][D + 1], g, sum);
        const float4v v = *reinterpret_cast<float4v*>(&jy[grp + e][d]);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = fmaf(v[i], g, y[i]);
      }
      if (last) {
        store_row(z, t, D, r, d, y, sum, top);
      } else {
        const int p = (slot_of(first) * z.R + r) * (D + 4) * 4;
        put4(parts_of, p + 4 * d, y);
        if (d == 0) put4(parts_of, p + 4 * D, float4v{top, sum, 0, 0});
      }
    }
  }
  if (last) break;
  count = z.count + 2 * kMaxShares + slot_of(0);
  step = g;
  n = groups;
  first = 0;
  }
  }
}

// The split of a call.  Everything here comes from the caller's sizes; the
// lengths themselves are on the device.
struct Plan {
  int tiles, shares, R;
  int64_t ids;
};

bool plan(const KvDev& c, const AttnCall& a, Plan* p) {
  const int64_t rows = (int64_t)a.max_q * (a.n_heads / c.H), tiles = (rows + 15) / 16, pairs = tiles * a.n_rows;
  p->ids = pairs * c.H;
  if (tiles > 65535 || p->ids > (1 << 23)) return false;   // what a grid holds
  p->tiles = (int)tiles;
  p->R = (int)(rows < 16 ? rows : 16);
  const int64_t room = (int64_t)c.max_pages * c.page_size;
  int64_t len = a.max_len > 0 ? a.max_len : room;
  if (a.window > 0 && len > (int64_t)a.window + a.max_q) len = (int64_t)a.window + a.max_q;
  const int64_t unit = 32 * kWaves, units = (len + unit - 1) / unit, slots = kCus * waves_of(c.D, c.G);
  p->shares = 0;
  // The line of units is counted in 31 bits, whatever the lengths are.
  if (pairs <= kMaxPairs && units > kMinUnits && (room / unit + 2) * p->ids < (1 << 30)) {
    const int64_t all = (units * p->ids + kUnitsOfShare - 1) / kUnitsOfShare;
    p->shares = (int)(all < slots ? all : slots);
  }
  return true;
}

// Two counts for each of the two parts that a share can leave.
constexpr size_t kCountBytes = TQ_WORKSPACE_COUNT_BYTES;
static_assert(4 * (2 + 2) * kMaxShares <= kCountBytes, "all counts at the front");

template <int D, int G>
void start(const Args& a, const Plan& p, hipStream_t s) {
  const dim3 grid = p.shares ? dim3(p.shares) : dim3(a.H, a.n_rows, p.tiles);
  kv_attn_kernel<D, G><<<grid, 64 * kWaves, 0, s>>>(a);
}

}  // namespace

bool kv_attention_plan(const KvDev& c, const AttnCall& a, size_t* ws_bytes) {
  Plan p;
  if (!plan(c, a, &p)) return false;
  *ws_bytes = p.shares > 0 ? kCountBytes + (size_t)2 * p.shares * p.R * (c.D + 4) * 4 : 0;
  return true;
}

hipError_t launch_kv_attention(const KvDev& c, int layer, const AttnCall& call, hipStream_t s) {
  Plan p;
  if (!plan(c, call, &p)) return hipErrorInvalidValue;
  Args a;
  a.layer = c.data + layer * c.layer_bytes;
  a.pages = c.pages;
  a.lens = c.lens;
  a.seqs = call.seqs;
  a.cu = call.cu;
  a.q = call.q.p;
  a.o = call.o;
  a.lse = call.lse;
  a.count = static_cast<int32_t*>(call.ws);
  a.part = call.ws != nullptr ? reinterpret_cast<float*>(static_cast<uint8_t*>(call.ws) + kCountBytes) : nullptr;
  a.q_ts = call.q.ts;
  a.q_hs = call.q.hs;
  a.page_bytes = c.page_bytes;
  a.scale_log2 = call.scale * 1.4426950408889634f;
  a.n_rows = call.n_rows;
  a.n_tokens = call.n_tokens;
  a.max_q = call.max_q;
  a.H = c.H;
  a.share = call.n_heads / c.H;
  a.share_magic = (uint32_t)((1ull << 32) / a.share + 1);
  a.window = call.window;
  a.page_shift = c.page_shift;
  a.n_seqs = c.n_seqs;
  a.max_pages = c.max_pages;
  a.n_pages = c.n_pages;
  a.tiles = p.tiles;
  a.shares = p.shares;
  a.R = p.R;
  a.out_f32 = call.out_f32;
  if (c.D == 64) {
    c.G == 32 ? start<64, 32>(a, p, s) : start<64, 64>(a, p, s);
  } else if (c.D == 128) {
    c.G == 32 ? start<128, 32>(a, p, s) : c.G == 64 ? start<128, 64>(a, p, s) : start<128, 128>(a, p, s);
  } else {
    c.G == 32 ? start<256, 32>(a, p, s) : c.G == 64 ? start<256, 64>(a, p, s) : start<256, 128>(a, p, s);
  }
  return hipGetLastError();
}

}  // namespace tq
