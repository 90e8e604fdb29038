// Attention over the 4-bit paged cache (gfx950), one pass over the keys and
// values with the running maximum and sum of the softmax:
//     s_j = scale * sum_g ( sk_jg (q . ck_j)_g + mk_jg sum_g q )
//     o   = sum_j ( p_j sv_jg ) cv_j  +  sum_j p_j mv_jg,   p_j = exp(s_j - max) / sum
// ck, cv: the codes less 8; sk, mk, sv, mv: scale and centred offset of token
// j's group g of channels.  No key or value is formed: the codes are exact
// operands of the matrix instructions and the parameters multiply the fp32
// sums (keys) or the probabilities (values).
//
// One wave takes records of 32 tokens against a tile of 16 QT query rows (a
// row is a query token and one of the heads that share the key/value head):
//   S^T = K Q^T: 16 tokens x 16 rows per instruction, a lane's four sums are
//   four tokens of the row lane % 16, and the eight it holds of a record are
//   its operand of the second product as they stand, since values are stored
//   with those eight tokens in one word: O^T += V^T P^T.
// A probability times a value scale enters as two fp16 numbers (hi + lo, 22
// bits); the sums of p, of p mv and of everything else are fp32.
//
// Work split: a workgroup has four waves that take the records of its range
// in turn and join their maxima, sums and outputs through LDS; a range is a
// part of the records that a tile of rows can see, so that few rows over a
// long cache fill the chip.  Parts leave their outputs in the workspace and
// a second launch joins them; where the caller's max_len makes one part the
// most there can be, it writes o itself.

#include "q4_internal.h"

namespace tq {
namespace {

constexpr int kWaves = 4;
constexpr float kLn2 = 0.69314718055994531f;

__device__ inline float4v mfma(half8 a, half8 b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

struct Args {
  const uint8_t* layer;    // the layer's pages
  const int32_t* pages;
  const int32_t* lens;
  const int32_t* seqs;
  const int32_t* cu;
  const uint16_t* q;
  void* o;
  float* lse;
  float* part;             // [tile][split][R][D + 2]: sums, maximum (log2), sum of p
  int64_t q_ts, q_hs, page_bytes;
  float scale_log2;
  int32_t n_rows, n_tokens, max_q, H, share, window;
  int32_t page_shift, n_seqs, max_pages, n_pages;
  int32_t tiles, splits, chunk;   // tiles of a row, parts of a tile, records of a part
  int32_t R;                      // rows of a tile kept in the workspace
  int32_t out_f32;
};

// What a tile of rows is: row b of the call, key/value head h, tile qt.
struct Tile {
  int b, h, qt;
  int seq, first, n, rows;   // slot, first token in q, tokens, rows of (b, h) in all
  int len;
  int row0;                  // first of the tile's rows
  int rec0, rec1, parts;     // records it can see, and in how many parts
};

template <int QT>
__device__ inline bool tile_of(const Args& a, int id, Tile* t) {
  t->h = id % a.H;
  t->b = id / a.H % a.n_rows;
  t->qt = id / a.H / a.n_rows;
  t->seq = a.seqs ? a.seqs[t->b] : t->b;
  int64_t first = a.cu ? a.cu[t->b] : t->b, end = a.cu ? a.cu[t->b + 1] : (int64_t)t->b + 1;
  const int64_t asked = end - first;
  const bool bad = first < 0 || asked < 0;
  end = min(min(end, (int64_t)a.n_tokens), first + a.max_q);
  t->first = (int)first;
  t->n = bad || end <= first ? 0 : (int)(end - first);
  t->rows = t->n * a.share;
  t->row0 = t->qt * 16 * QT;
  if (t->row0 >= t->rows) return false;
  t->len = 0;
  if (t->seq >= 0 && t->seq < a.n_seqs)
    t->len = (int)min(min(max((int64_t)a.lens[t->seq], (int64_t)0), (int64_t)a.max_pages << a.page_shift),
                      (int64_t)INT32_MAX - 64);
  // Position of query token i is base + i; all of what was asked for counts.
  const int64_t base = t->len - asked;
  const int i0 = t->row0 / a.share, i1 = min(t->row0 + 16 * QT - 1, t->rows - 1) / a.share;
  const int64_t hi = min((int64_t)t->len, base + i1 + 1);
  const int64_t lo = a.window > 0 ? max((int64_t)0, base + i0 + 1 - a.window) : 0;
  t->rec0 = (int)(lo >> 5);
  t->rec1 = hi > lo ? (int)((hi + 31) >> 5) : t->rec0;
  t->parts = min(a.splits, max(1, (t->rec1 - t->rec0 + a.chunk - 1) / a.chunk));
  return true;
}

// Everything of a record that a lane needs, as it lies in memory.
template <int D, int G>
struct Record {
  uint32_t k[2][D / 32];
  u4v v[D / 64];
  u4v kp[D / G][2], vp[D / G][2];
};

template <int D, int G, int QT>
__global__ void __launch_bounds__(64 * kWaves) kv_attn_kernel(Args a) {
  constexpr int NG = D / G, J = G / 32, KD = D / 32, VD = D / 16;
  constexpr int64_t kRec = 32 * (D + 8 * NG);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane >> 4, col = lane & 15;
  const int tiles = a.H * a.n_rows * a.tiles;
  const int part = blockIdx.x / tiles, id = blockIdx.x % tiles;
  Tile t;
  if (!tile_of<QT>(a, id, &t) || part >= t.parts) return;
  const int rec0 = t.rec0 + part * a.chunk;
  const int rec1 = part == t.parts - 1 ? t.rec1 : rec0 + a.chunk;

  // The lane's query rows as operands, their sums per group, their positions.
  half8 q[QT][KD];
  float qs[QT][NG];
  int pos[QT];
  const int64_t base = (int64_t)t.len - (a.cu ? (int64_t)a.cu[t.b + 1] - a.cu[t.b] : 1);
  const half8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
  for (int u = 0; u < QT; ++u) {
    const int row = t.row0 + 16 * u + col;
    const bool in = row < t.rows;
    const int tok = in ? row / a.share : 0, head = in ? t.h * a.share + row % a.share : 0;
    const uint16_t* qp = a.q + (int64_t)(t.first + tok) * a.q_ts + head * a.q_hs;
    pos[u] = in ? (int)max(base + tok, (int64_t)-1) : -1;
#pragma unroll
    for (int j = 0; j < KD; ++j) q[u][j] = in ? load8(qp + 32 * j + 8 * c) : zero;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      float s = 0.0f;
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) s += (float)q[u][g * J + j][e];
      s += __shfl_xor(s, 16);
      s += __shfl_xor(s, 32);
      qs[u][g] = s * a.scale_log2;
    }
  }
  // The positions between which every row of the tile sees every token.
  int all0 = 0, all1;
  {
    const int i0 = t.row0 / a.share, i1 = min(t.row0 + 16 * QT - 1, t.rows - 1) / a.share;
    all1 = (int)max((int64_t)0, min((int64_t)t.len, base + i0 + 1));
    if (a.window > 0) all0 = (int)max((int64_t)0, base + i1 + 1 - a.window);
  }

  float4v acc[QT][VD];
  float macc[QT][NG], m[QT], l[QT];
#pragma unroll
  for (int u = 0; u < QT; ++u) {
    m[u] = -__builtin_inff();
    l[u] = 0.0f;
#pragma unroll
    for (int g = 0; g < NG; ++g) macc[u][g] = 0.0f;
#pragma unroll
    for (int j = 0; j < VD; ++j) acc[u][j] = float4v{0, 0, 0, 0};
  }

  // The page of a record, -1 where there is none.
  const int per_shift = a.page_shift - 5;
  const int32_t* row_pages = a.pages + (int64_t)(t.len > 0 ? t.seq : 0) * a.max_pages;
  auto page_at = [&](int rec) {
    const int p = row_pages[rec >> per_shift];
    return p >= 0 && p < a.n_pages ? p : -1;
  };
  auto load = [&](Record<D, G>& r, int rec, int page) {
    const int per = 1 << per_shift;
    const uint8_t* p = a.layer + (int64_t)page * a.page_bytes + ((int64_t)t.h * per + (rec & (per - 1))) * kRec;
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
#pragma unroll
    for (int i = 0; i < D / 64; ++i) r.v[i] = *reinterpret_cast<const u4v*>(p + 16 * D + (64 * i + lane) * 16);
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        r.kp[g][h] = *reinterpret_cast<const u4v*>(p + 32 * D + g * 128 + (16 * h + 4 * c) * 4);
        r.vp[g][h] = *reinterpret_cast<const u4v*>(p + 32 * D + (NG + g) * 128 + (16 * h + 4 * c) * 4);
      }
  };

  auto compute = [&](const Record<D, G>& r, int rec) {
    const bool whole = rec * 32 >= all0 && rec * 32 + 32 <= all1;
    half8 kf[2][KD];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < KD; ++j) kf[h][j] = code_operand(r.k[h][j]);
    half8 hi[QT][NG], lo[QT][NG];
#pragma unroll
    for (int u = 0; u < QT; ++u) {
      float s[2][4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float x[4] = {0, 0, 0, 0}, y[4] = {0, 0, 0, 0};
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          float4v z = {0, 0, 0, 0};
#pragma unroll
          for (int j = 0; j < J; ++j) z = mfma(kf[h][g * J + j], q[u][g * J + j], z);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float sk = lo_half(r.kp[g][h][i]);
            x[i] = fmaf(sk, z[i], x[i]);
            y[i] = fmaf(centred(sk, hi_half(r.kp[g][h][i])), qs[u][g], y[i]);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) s[h][i] = fmaf(x[i], a.scale_log2, y[i]);
      }
      uint32_t seen = 0xFFu;
      if (!whole) {
        seen = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int at = rec * 32 + 16 * h + 4 * c + i;
            const bool see = at <= pos[u] && (a.window <= 0 || at > pos[u] - a.window);
            seen |= (uint32_t)see << (4 * h + i);
            if (!see) s[h][i] = -__builtin_inff();
          }
      }
      float top = s[0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top = fmaxf(top, s[i >> 2][i & 3]);
      if (__builtin_amdgcn_ballot_w64(top > m[u]) != 0) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float now = fmaxf(top, m[u]);
        const float f = now == -__builtin_inff() ? 1.0f : exp2f(m[u] - now);
        m[u] = now;
        l[u] *= f;
#pragma unroll
        for (int g = 0; g < NG; ++g) macc[u][g] *= f;
#pragma unroll
        for (int j = 0; j < VD; ++j) acc[u][j] *= f;
      }
      const float ref = m[u] == -__builtin_inff() ? 0.0f : m[u];
      float p[2][4];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[h][i] = __builtin_amdgcn_exp2f(s[h][i] - ref);
          l[u] += p[h][i];
        }
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        float w[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float sv = lo_half(r.vp[g][h][i]), mv = centred(sv, hi_half(r.vp[g][h][i]));
            if (!whole && !((seen >> (4 * h + i)) & 1)) sv = mv = 0.0f;   // what no row may see may be anything
            w[h][i] = p[h][i] * sv;
            macc[u][g] = fmaf(p[h][i], mv, macc[u][g]);
          }
        // Operand register i: tokens 4c + i and 16 + 4c + i.
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const _Float16 x = (_Float16)w[h][i];
            hi[u][g][2 * i + h] = x;
            lo[u][g][2 * i + h] = (_Float16)(w[h][i] - (float)x);
          }
      }
    }
#pragma unroll
    for (int j = 0; j < VD; ++j) {
      const half8 vf = code_operand(r.v[j >> 2][j & 3]);
#pragma unroll
      for (int u = 0; u < QT; ++u) {
        acc[u][j] = mfma(vf, hi[u][j * 16 / G], acc[u][j]);
        acc[u][j] = mfma(vf, lo[u][j * 16 / G], acc[u][j]);
      }
    }
  };

  if constexpr (D == 256) {
    for (int rec = rec0 + wave; rec < rec1; rec += kWaves) {
      const int page = page_at(rec);
      if (page < 0) continue;
      Record<D, G> cur;
      load(cur, rec, page);
      compute(cur, rec);
    }
  } else {
    Record<D, G> cur, nxt;
    int rec = rec0 + wave, page = -1, page_n = -1;
    if (rec < rec1) {
      page = page_at(rec);
      if (page >= 0) load(cur, rec, page);
    }
    while (rec < rec1) {
      const int next = rec + kWaves;
      if (next < rec1) {
        page_n = page_at(next);
        if (page_n >= 0) load(nxt, next, page_n);
      }
      if (page >= 0) compute(cur, rec);
      cur = nxt;
      page = page_n;
      rec = next;
    }
  }

  // Join the four lane groups' sums, then the waves.
  __shared__ float sm[kWaves][16], sl[kWaves][16];
  __shared__ float so[kWaves][16][D + 4];
#pragma unroll
  for (int u = 0; u < QT; ++u) {
    float L = l[u];
    L += __shfl_xor(L, 16);
    L += __shfl_xor(L, 32);
    float M[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      M[g] = macc[u][g] + __shfl_xor(macc[u][g], 16);
      M[g] += __shfl_xor(M[g], 32);
    }
    if (u > 0) __syncthreads();
    if (c == 0) sm[wave][col] = m[u];
    __syncthreads();
    float top = sm[0][col];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, sm[w][col]);
    const float f = m[u] == -__builtin_inff() ? 0.0f : exp2f(m[u] - top);
    if (c == 0) sl[wave][col] = L * f;
#pragma unroll
    for (int j = 0; j < VD; ++j) {
      float4v y;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = (acc[u][j][i] + M[j * 16 / G]) * f;
      *reinterpret_cast<float4v*>(&so[wave][col][16 * j + 4 * c]) = y;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * D / 4; i += 64 * kWaves) {
      const int r = i / (D / 4), d = i % (D / 4) * 4, row = t.row0 + 16 * u + r;
      if (row >= t.rows) continue;
      float4v y = *reinterpret_cast<float4v*>(&so[0][r][d]);
      float sum = sl[0][r], most = sm[0][r];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) {
        y += *reinterpret_cast<float4v*>(&so[w][r][d]);
        sum += sl[w][r];
        most = fmaxf(most, sm[w][r]);
      }
      if (t.parts > 1) {
        float* p = a.part + (((int64_t)id * a.splits + part) * a.R + 16 * u + r) * (D + 4);
        *reinterpret_cast<float4v*>(p + d) = y;
        if (d == 0) {
          p[D] = most;
          p[D + 1] = sum;
        }
        continue;
      }
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
      const int64_t at = (int64_t)(t.first + row / a.share) * (a.H * a.share) + t.h * a.share + row % a.share;
      y *= inv;
      if (a.out_f32) {
        *reinterpret_cast<float4v*>(static_cast<float*>(a.o) + at * D + d) = y;
      } else {
        const half4 z = {(_Float16)y[0], (_Float16)y[1], (_Float16)y[2], (_Float16)y[3]};
        *reinterpret_cast<half4*>(static_cast<uint16_t*>(a.o) + at * D + d) = z;
      }
      if (a.lse && d == 0) a.lse[at] = sum == 0.0f ? -__builtin_inff() : (most + log2f(sum)) * kLn2;
    }
  }
}

// Joins the parts of a tile's rows: a wave per row.
template <int D, int QT>
__global__ void __launch_bounds__(256) kv_join_kernel(Args a) {
  const int id = blockIdx.x, r = blockIdx.y * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  Tile t;
  if (!tile_of<QT>(a, id, &t) || t.parts == 1) return;
  const int row = t.row0 + r;
  if (r >= 16 * QT || row >= t.rows) return;
  const float* p = a.part + ((int64_t)id * a.splits * a.R + r) * (D + 4);
  const int64_t step = (int64_t)a.R * (D + 4);
  float top = -__builtin_inff();
  for (int s = lane; s < t.parts; s += 64) top = fmaxf(top, p[s * step + D]);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  float sum = 0.0f, y[D / 64];
#pragma unroll
  for (int e = 0; e < D / 64; ++e) y[e] = 0.0f;
  for (int s = 0; s < t.parts; ++s) {
    const float m = p[s * step + D];
    const float f = m == -__builtin_inff() ? 0.0f : exp2f(m - top);
    sum = fmaf(p[s * step + D + 1], f, sum);
#pragma unroll
    for (int e = 0; e < D / 64; ++e) y[e] = fmaf(p[s * step + 64 * e + lane], f, y[e]);
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  const int64_t at = (int64_t)(t.first + row / a.share) * (a.H * a.share) + t.h * a.share + row % a.share;
#pragma unroll
  for (int e = 0; e < D / 64; ++e) {
    if (a.out_f32)
      static_cast<float*>(a.o)[at * D + 64 * e + lane] = y[e] * inv;
    else
      static_cast<_Float16*>(a.o)[at * D + 64 * e + lane] = (_Float16)(y[e] * inv);
  }
  if (a.lse && lane == 0) a.lse[at] = sum == 0.0f ? -__builtin_inff() : (top + log2f(sum)) * kLn2;
}

// The split of a call.  Everything here comes from the caller's sizes; the
// lengths themselves are on the device.
struct Plan {
  int qt, tiles, splits, chunk, R;
  int64_t ids;
};

bool plan(const KvDev& c, const AttnCall& a, Plan* p) {
  const int64_t share = a.n_heads / c.H, rows = (int64_t)a.max_q * share;
  // More rows a tile would not fit the registers: 4 tiles of 16 at D = 64, 2
  // at D = 128, 1 at D = 256, where the next record is not fetched ahead
  // either.  No variant spills: one that did gave wrong sums.
  const int most = 256 / c.D;
  p->qt = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  if (p->qt > most) p->qt = most;
  const int64_t tiles = (rows + 16 * p->qt - 1) / (16 * p->qt);
  p->ids = tiles * c.H * a.n_rows;
  if (p->ids > (1 << 23)) return false;   // a launch has fewer than 2^32 threads
  p->tiles = (int)tiles;
  p->R = (int)(rows < 16 * p->qt ? rows : 16 * p->qt);
  int64_t len = a.max_len > 0 ? a.max_len : (int64_t)c.max_pages * c.page_size;
  if (a.window > 0 && len > (int64_t)a.window + a.max_q) len = (int64_t)a.window + a.max_q;
  const int64_t recs = (len + 31) / 32 + 1;
  // Parts of 16 records (four a wave) at least, and no more workgroups than
  // about 2048.
  int64_t splits = (2048 + p->ids - 1) / p->ids;
  if (splits > (recs + 15) / 16) splits = (recs + 15) / 16;
  if (splits < 1) splits = 1;
  if (splits > 1024) splits = 1024;
  p->splits = (int)splits;
  p->chunk = (int)((recs + splits - 1) / splits);
  return true;
}

template <int D, int G, int QT>
void start(const Args& a, const Plan& p, hipStream_t s) {
  kv_attn_kernel<D, G, QT><<<(uint32_t)(p.ids * p.splits), 64 * kWaves, 0, s>>>(a);
  if (p.splits > 1) kv_join_kernel<D, QT><<<dim3((uint32_t)p.ids, (p.R + 3) / 4), 256, 0, s>>>(a);
}

template <int D, int G>
void start_qt(const Args& a, const Plan& p, hipStream_t s) {
  if (p.qt == 1) start<D, G, 1>(a, p, s);
  if constexpr (D <= 128)
    if (p.qt == 2) start<D, G, 2>(a, p, s);
  if constexpr (D == 64)
    if (p.qt == 4) start<D, G, 4>(a, p, s);
}

}  // namespace

bool kv_attention_plan(const KvDev& c, const AttnCall& a, size_t* ws_bytes) {
  Plan p;
  if (!plan(c, a, &p)) return false;
  *ws_bytes = p.splits > 1 ? (size_t)(p.ids * p.splits * p.R) * (c.D + 4) * 4 : 0;
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
  a.part = static_cast<float*>(call.ws);
  a.q_ts = call.q.ts;
  a.q_hs = call.q.hs;
  a.page_bytes = c.page_bytes;
  a.scale_log2 = call.scale * 1.4426950408889634f;
  a.n_rows = call.n_rows;
  a.n_tokens = call.n_tokens;
  a.max_q = call.max_q;
  a.H = c.H;
  a.share = call.n_heads / c.H;
  a.window = call.window;
  a.page_shift = c.page_shift;
  a.n_seqs = c.n_seqs;
  a.max_pages = c.max_pages;
  a.n_pages = c.n_pages;
  a.tiles = p.tiles;
  a.splits = p.splits;
  a.chunk = p.chunk;
  a.R = p.R;
  a.out_f32 = call.out_f32;
  if (c.D == 64) {
    c.G == 32 ? start_qt<64, 32>(a, p, s) : start_qt<64, 64>(a, p, s);
  } else if (c.D == 128) {
    c.G == 32 ? start_qt<128, 32>(a, p, s) : c.G == 64 ? start_qt<128, 64>(a, p, s) : start_qt<128, 128>(a, p, s);
  } else {
    c.G == 32 ? start_qt<256, 32>(a, p, s) : c.G == 64 ? start_qt<256, 64>(a, p, s) : start_qt<256, 128>(a, p, s);
  }
  return hipGetLastError();
}

}  // namespace tq
