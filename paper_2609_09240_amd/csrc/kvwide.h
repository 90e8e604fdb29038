// Attention of many query rows over the same records of the 4-bit cache (gfx950):
// the queries of a group of rows over the tokens that they share, and those of a
// chunk over its window and sinks.  The mathematics are those of
// kvattn_kernel.h, and so are the roundings.
//
// Four waves take RT tiles of 16 rows each over the same records.  A record is
// unpacked once for all of them: every thread turns its words of codes into
// operands of the matrix instructions and leaves them in LDS, where a wave reads
// each operand once for its RT tiles.  Two records are in LDS, and the one after
// them is on its way: one barrier a record.
#pragma once

#include "kvattn_kernel.h"

namespace tq {
namespace {

constexpr int wide_waves(int D, int G, int RT) { return D == 256 ? 1 : RT == 2 ? 2 : D == 64 ? 4 : G == 32 ? 2 : 3; }

// A record in LDS: operands by lane, keys [2][KD] and values [VD], and the
// parameters: pairs of the keys [NG][32], scales of the values [NG][32], and their
// offsets with 8 scales [NG][32].
template <int D, int G>
struct Stage {
  half8 k[2][D / 32][64];
  half8 v[D / 16][64];
  float vm[D / G][32];
  uint32_t kp[D / G][32];
  uint16_t vs[D / G][32];
};

template <int D, int G, int MODE, int RT>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(wide_waves(D, G, RT))))
kv_wide_kernel(MoreArgs args) {
  constexpr int NG = D / G, J = G / 32, KD = D / 32, VD = D / 16, R = 64 * RT;
  constexpr int64_t kRec = 32 * (D + 8 * NG);
  constexpr int kWords = D / 32, kLoads = kWords >= 4 ? kWords / 4 : 1;   // words of codes a thread, 16 bytes a load
  __shared__ Stage<D, G> stage[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane >> 4, col = lane & 15;
  auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  Tile t;
  // A workgroup is a head, a part of the records, and a tile of a row or group.
  const MoreArgs& a = args;
  const int h = blockIdx.x % a.H, part = blockIdx.x / a.H, parts = MODE == kShared ? a.stack_parts : a.parts;
  if constexpr (MODE == kShared) {
    if (!stack_of<R>(a, blockIdx.y, blockIdx.z, &t)) return;
  } else {
    if (!tile_of<MODE, R>(a, blockIdx.y, blockIdx.z, &t)) return;
  }
  t.h = h;
  const int64_t all = t.rec1 - t.rec0;
  int rec0 = t.rec0 + (int)(all * part / parts), rec1 = t.rec0 + (int)(all * (part + 1) / parts);
  rec0 = uniform(rec0);
  rec1 = uniform(rec1);
  t.rows = uniform(t.rows);
  t.row0 = uniform(t.row0);
  t.tok0 = uniform(t.tok0);
  t.head0 = uniform(t.head0);
  t.first = uniform(t.first);
  t.n = uniform(t.n);
  t.len = uniform(t.len);
  int v0 = 0, win0 = 0;
  if constexpr (MODE == kSinks) {
    v0 = uniform(t.rec0);
    win0 = uniform(t.win0);
  }
  auto in_slot = [&](int rec) { return MODE == kSinks && rec < win0 ? rec - v0 : rec; };
  const int per_shift = a.page_shift - 5;
  const table_ptr row_pages = as_table(a.pages) + (int64_t)(t.len > 0 ? t.seq : 0) * a.max_pages;
  // The page of a record, and the bytes of a record: one that is not there (no
  // page, or behind the last one) is not looked at, and the layer's first in
  // its place.
  auto page_of = [&](int rec) { return row_pages[in_slot(min(rec, rec1 - 1)) >> per_shift]; };
  auto there = [&](int rec, int page) { return rec < rec1 && page >= 0 && page < a.n_pages; };
  auto bytes_of = [&](int rec, int page) {
    const int per = 1 << per_shift, in = in_slot(rec) & (per - 1);
    return a.layer + (there(rec, page) ? (int64_t)page * a.page_bytes + ((int64_t)h * per + in) * kRec : 0);
  };

  // What a thread loads of a record: its words of codes, one word of parameters.
  u4v codes[kLoads];
  uint32_t param[NG > 4 ? 2 : 1];
  auto load = [&](const uint8_t* p) {
    if constexpr (D == 64) {
      const u2v x = *reinterpret_cast<const u2v*>(p + 8 * tid);
      codes[0] = u4v{x[0], x[1], 0, 0};
    } else {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) codes[i] = *reinterpret_cast<const u4v*>(p + (256 * i + tid) * 16);
    }
#pragma unroll
    for (int i = 0; i < (NG > 4 ? 2 : 1); ++i)
      param[i] = *reinterpret_cast<const uint32_t*>(p + 32 * D + 4 * ((tid + 256 * i) % (64 * NG)));
  };
  // Word w of a record's codes goes to this place.
  auto store = [&](Stage<D, G>& s) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
#pragma unroll
      for (int e = 0; e < (D == 64 ? 2 : 4); ++e) {
        const int w = D == 64 ? 2 * tid + e : (256 * i + tid) * 4 + e;
        const half8 x = code_operand(codes[i][e]);
        if (w < 4 * D)
          s.k[w / (64 * KD)][w % KD][w / KD % 64] = x;
        else
          s.v[(w - 4 * D) / 256 * 4 + w % 4][(w - 4 * D) / 4 % 64] = x;
      }
#pragma unroll
    for (int i = 0; i < (NG > 4 ? 2 : 1); ++i) {
      const int w = tid + 256 * i;
      if (w < 32 * NG) {
        s.kp[w / 32][w % 32] = param[i];
      } else if (w < 64 * NG) {
        const half2v x = pair(param[i]);
        s.vs[w / 32 - NG][w % 32] = (uint16_t)param[i];
        s.vm[w / 32 - NG][w % 32] = fmaf(8.0f, (float)x[0], (float)x[1]);
      }
    }
  };

  // Pages of the records n, n + 1 and n + 2; n + 1 is on its way.
  int page0 = 0, page1 = 0, page2 = 0;
  if (rec0 < rec1) {
    page0 = page_of(rec0);
    page1 = page_of(rec0 + 1);
    page2 = page_of(rec0 + 2);
    load(bytes_of(rec0, page0));
  }

  // Queries as operands, their sums per group, positions: as in kvattn_kernel.h.
  half8 q[RT][KD];
  float qs[RT][NG];
  int pos[RT], all0[RT], all1[RT], any0[RT], any1[RT];
  const int64_t base = (int64_t)t.len - t.asked;
  const half8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int row = (wave * RT + r) * 16 + col;
    const bool in = t.row0 + row < t.rows;
    const int up = by_share(a, t.head0 + row), tok = in ? t.tok0 + up : 0;
    const int head = in ? h * a.share + t.head0 + row - up * a.share : 0;
    const uint16_t* qp = a.q + (int64_t)(t.first + tok) * a.q_ts + head * a.q_hs;
    pos[r] = -1;
    if (in) {
      if constexpr (MODE == kShared)
        pos[r] = stack_pos(a, t.b, t.b1, t.first + tok);
      else
        pos[r] = (int)max(base + tok, (int64_t)-1);
    }
#pragma unroll
    for (int j = 0; j < KD; ++j) q[r][j] = in ? load8(qp + 32 * j + 8 * c) : zero;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      float s = 0.0f;
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) s += (float)q[r][g * J + j][e];
      s += __shfl_xor(s, 16);
      s += __shfl_xor(s, 32);
      qs[r][g] = s / kCodeUnit;
    }
    // The positions that all rows of the tile see, and those that some do.
    // (Tokens that a group's call leaves out are not taken up, whatever they get.)
    int least = in && (MODE != kShared || pos[r] >= 0) ? pos[r] : INT32_MAX, most = pos[r];
#pragma unroll
    for (int k = 1; k < 16; k *= 2) {
      least = min(least, __shfl_xor(least, k));
      most = max(most, __shfl_xor(most, k));
    }
    all0[r] = any0[r] = 0;
    if (MODE == kSinks && most >= 0) {
      all0[r] = max(0, most + 1 - a.window);
      any0[r] = max(0, least + 1 - a.window);
    }
    all0[r] = uniform(all0[r]);
    any0[r] = uniform(any0[r]);
    all1[r] = uniform(min(least, most) + 1);
    any1[r] = uniform(most + 1);
  }

  const float logit = a.scale_log2 * kCodeUnit;
  const float kNone = -3.0e38f;
  float4v acc[RT][VD];
  float macc[RT][NG], per_unit[RT][NG], ref[RT], grow[RT], l[RT], unit2[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    unit2[r] = 0x1p-23f;
    ref[r] = 0.0f;
    grow[r] = kNone;
    l[r] = 0.0f;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      macc[r][g] = 0.0f;
      per_unit[r][g] = 1.0f;
    }
#pragma unroll
    for (int j = 0; j < VD; ++j) acc[r][j] = float4v{0, 0, 0, 0};
  }

  if (rec0 < rec1) {
    store(stage[0]);
    load(bytes_of(rec0 + 1, page1));
  }
  for (int rec = rec0, now = 0; rec < rec1; ++rec, now ^= 1) {
    __syncthreads();   // the record is there, and nobody reads the other place
    const int t0 = 32 * in_slot(rec);
    const Stage<D, G>& st = stage[now];
    // The first operands, then the next record's place while they come.
    half8 kf[KD];
    u4v kp[NG];
    auto keys = [&](int hf) {
#pragma unroll
      for (int j = 0; j < KD; ++j) kf[j] = st.k[hf][j][lane];
#pragma unroll
      for (int g = 0; g < NG; ++g) kp[g] = *reinterpret_cast<const u4v*>(&st.kp[g][16 * hf + 4 * c]);
    };
    keys(0);
    bool see[RT], whole[RT], work = false;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      whole[r] = t0 >= all0[r] && t0 + 32 <= all1[r];
      see[r] = t0 < any1[r] && t0 + 32 > any0[r];
      if constexpr (MODE == kSinks) {
        whole[r] |= t0 + 32 <= min(a.sinks, all1[r]);
        see[r] |= t0 < a.sinks && t0 < any1[r];
      }
      work |= see[r];
    }
    work &= there(rec, page0);
    store(stage[now ^ 1]);
    load(bytes_of(rec + 2, page2));
    page0 = page1;
    page1 = page2;
    page2 = page_of(rec + 3);
    if (work) {
      float s[RT][2][4];
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        if (hf == 1) keys(1);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          float x[4] = {0, 0, 0, 0};
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            const float q8 = 8.0f * qs[r][g];
            float4v z = {q8, q8, q8, q8};
#pragma unroll
            for (int j = 0; j < J; ++j) z = mfma(kf[g * J + j], q[r][g * J + j], z);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const half2v p = pair(kp[g][i]);
              x[i] = fmaf((float)p[0], z[i], x[i]);
              x[i] = fmaf((float)p[1], qs[r][g], x[i]);
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) s[r][hf][i] = fmaf(x[i], logit, -ref[r]);
        }
      }
      u2v vs[NG][2];
      float4v vm[NG][2];
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          vs[g][hf] = *reinterpret_cast<const u2v*>(&st.vs[g][16 * hf + 4 * c]);
          vm[g][hf] = *reinterpret_cast<const float4v*>(&st.vm[g][16 * hf + 4 * c]);
        }
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        u4v hi[NG], lo[NG];
        u2v ws[NG][2];
        float4v wm[NG][2];
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            ws[g][hf] = vs[g][hf];
            wm[g][hf] = vm[g][hf];
          }
        if (!whole[r]) {
          asm volatile("");   // a branch, not selects
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int tok = t0 + 16 * hf + 4 * c + i;
              bool ok = tok <= pos[r];
              if constexpr (MODE == kSinks) ok &= tok > pos[r] - a.window || tok < a.sinks;
              if (!ok) s[r][hf][i] = -__builtin_inff();
#pragma unroll
              for (int g = 0; g < NG; ++g) {   // what is not seen may be anything
                ws[g][hf][i / 2] = ok ? ws[g][hf][i / 2] : ws[g][hf][i / 2] & (i & 1 ? 0x0000FFFFu : 0xFFFF0000u);
                wm[g][hf][i] = ok ? wm[g][hf][i] : 0.0f;
              }
            }
        }
        float top = fmaxf(fmaxf(fmaxf(s[r][0][0], s[r][0][1]), fmaxf(s[r][0][2], s[r][0][3])),
                          fmaxf(fmaxf(s[r][1][0], s[r][1][1]), fmaxf(s[r][1][2], s[r][1][3])));
        auto begun = [&] { return __builtin_amdgcn_ballot_w64(l[r] != 0.0f) != 0; };
        if (__builtin_amdgcn_ballot_w64(top > grow[r]) != 0) {
          top = __builtin_bit_cast(float, over_row(__builtin_bit_cast(uint32_t, top), [](uint32_t a, uint32_t b) {
            return __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)));
          }));
          const bool some = begun();
          if (top > grow[r]) {
            const float set = kHighSet - log2_of(0.5f * unit2[r]), by = top - set;
            if (some) {
              const float f = grow[r] == kNone ? 0.0f : exp2f(-by);
              l[r] *= f;
#pragma unroll
              for (int g = 0; g < NG; ++g) macc[r][g] *= f;
#pragma unroll
              for (int j = 0; j < VD; ++j) acc[r][j] *= f;
            }
            ref[r] += by;
            grow[r] = set + (kHigh - kHighSet);
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
#pragma unroll
              for (int i = 0; i < 4; ++i) s[r][hf][i] -= by;
          }
        }
        // The largest scale of a group among the tokens that the row sees, as a whole number.
        uint32_t most[NG];
        float big = 0.0f;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          const uint32_t x = larger(larger(ws[g][0][0], ws[g][0][1]), larger(ws[g][1][0], ws[g][1][1]));
          most[g] = larger(x, x >> 16);
          big = fmaxf(big, fmaf(lo_half(most[g]), per_unit[r][g], 0.0f));
        }
        if (__builtin_amdgcn_ballot_w64(big >= unit2[r]) != 0) {
          const float unit0 = 0.5f * unit2[r];
          const bool some = begun();
          float now0 = unit0;
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            const uint32_t x = over_row(most[g], larger);
            const float unit = unit0 * over_power(per_unit[r][g]), scale = lo_half(x);
            const float now = scale >= 2.0f * unit ? power_of(scale) : unit;
            if (g == 0) now0 = now;
            per_unit[r][g] = now0 * over_power(now);
            const float f = unit * over_power(now);
            if (some)
#pragma unroll
              for (int j = g * G / 16; j < (g + 1) * G / 16; ++j) acc[r][j] *= f;
          }
          const float f = unit0 * over_power(now0), by = -log2_of(f);
          unit2[r] = 2.0f * now0;
          if (some) {
            l[r] *= f;
#pragma unroll
            for (int g = 0; g < NG; ++g) macc[r][g] *= f;
          }
          ref[r] += by;
          grow[r] -= by;   // kNone stays what it is
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[r][hf][i] -= by;
        }
        float p[2][4];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            p[hf][i] = __builtin_amdgcn_exp2f(s[r][hf][i]);
            l[r] += p[hf][i];
          }
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float w[2];
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              const half2v v = pair(ws[g][hf][i / 2]);
              w[hf] = fmaf(g == 0 ? p[hf][i] : p[hf][i] * per_unit[r][g], (float)v[i & 1], 0x1p-25f);
              macc[r][g] = fmaf(p[hf][i], wm[g][hf][i], macc[r][g]);
            }
            const uint32_t x = cut(w[0], w[1]);
            hi[g][i] = x;
            lo[g][i] = cut(rest0(x, w[0]), rest1(x, w[1]));
          }
        // (Operands read for both tiles at once would hold both tiles' probabilities,
        // which do not fit the registers.)
#pragma unroll
        for (int j0 = 0; j0 < VD; j0 += 4) {
          half8 vf[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) vf[j] = st.v[j0 + j][lane];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[r][j0 + j] = mfma(vf[j], __builtin_bit_cast(half8, hi[(j0 + j) * 16 / G]), acc[r][j0 + j]);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[r][j0 + j] = mfma(vf[j], __builtin_bit_cast(half8, lo[(j0 + j) * 16 / G]), acc[r][j0 + j]);
        }
      }
    }
  }

  // Join the four lane groups' sums.
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int row = (wave * RT + r) * 16 + col;
    const float m = grow[r] == kNone ? -__builtin_inff() : ref[r];
    float L = l[r];
    L += __shfl_xor(L, 16);
    L += __shfl_xor(L, 32);
    float M[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      M[g] = macc[r][g] + __shfl_xor(macc[r][g], 16);
      M[g] += __shfl_xor(M[g], 32);
    }
    if (t.row0 + row >= t.rows) continue;
#pragma unroll
    for (int j = 0; j < VD; ++j) {
      float4v y;
      const float unit = kCodeUnit / per_unit[r][j * 16 / G];
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = fmaf(acc[r][j][i], unit, M[j * 16 / G]);
      if (MODE == kSinks && parts == 1)
        store_row(a, t, D, row, 16 * j + 4 * c, y, L, m);
      else
        store_part(a, t, D, row, 16 * j + 4 * c, y, L, m, part);
    }
  }
}

}  // namespace
}  // namespace tq
