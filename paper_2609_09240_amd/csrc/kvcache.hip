// Writing and reading the 4-bit key/value cache (gfx950).
//
// A workgroup owns one record: 32 tokens of one head of one row of the call.
// Keys go to their words straight from the thread that quantised them (8
// channels of a token are one word); values cross over LDS, because a word
// of theirs holds 8 tokens of one channel.  A word that also holds tokens
// that are not new is read, changed and written back by one thread.
//
// 6000 tokens of 8 heads of 128 in groups of 32 (24.6 MB in, 7.7 MB out): 14.9
// us, 2.2 TB/s (13.8 at best), read back 13.2 us, 2.4 TB/s.  Neither is at a
// bound: the copy rate is 4.9 TB/s, the arithmetic takes 59 and 48 % of the
// vector slots (a division a value took 1.5 times as long).  What is left in the
// code: value words go out 16 bytes apart, and reading back divides by three
// run-time numbers for every 8 channels and reads a word of LDS a value.  One
// token each of 64 rows: 5.7 and 4.2 us, the launch and three trips to memory
// one after the other.

#include "q4_internal.h"

namespace tq {
namespace {

// Row i's part of a call: its slot, where its tokens start in the call and in
// the slot, and how many there are.
struct Row {
  int seq, first, start, n;
  bool over;   // the call asked for more than it may write
};

__device__ inline Row row_of(const KvDev& c, const int32_t* seqs, const int32_t* starts, const int32_t* cu, int i,
                             int n_tokens, int max_new) {
  Row r;
  r.seq = seqs ? seqs[i] : i;
  r.start = starts[i];
  int64_t first = cu ? cu[i] : i, end = cu ? cu[i + 1] : (int64_t)i + 1;
  r.over = false;
  if (first < 0) { first = 0; r.over = true; }
  if (end > n_tokens) { end = n_tokens; r.over = true; }
  if (end - first > max_new) { end = first + max_new; r.over = true; }
  r.first = (int)first;
  r.n = end > first ? (int)(end - first) : 0;
  return r;
}

// The record `rec` of head h of slot seq in `layer`; null where no page is.
__device__ inline uint8_t* record(const KvDev& c, int layer, int seq, int64_t rec, int h) {
  const int per = c.page_size >> 5;
  const int64_t slot = rec >> (c.page_shift - 5);
  if (slot >= c.max_pages) return nullptr;
  const int page = c.pages[(int64_t)seq * c.max_pages + slot];
  if (page < 0 || page >= c.n_pages) return nullptr;
  const int64_t at = (int64_t)h * per + (rec & (per - 1));
  return c.data + layer * c.layer_bytes + page * c.page_bytes + at * kv_record_bytes(c.D, c.G);
}

// Smallest and largest of a group over the `per` neighbouring lanes that hold
// it, and whether all of it is finite.
template <int per>
__device__ __forceinline__ void reduce_group(float* lo, float* hi, int* f) {
#pragma unroll
  for (int d = 1; d < per; d <<= 1) {
    *lo = fminf(*lo, __shfl_xor(*lo, d));
    *hi = fmaxf(*hi, __shfl_xor(*hi, d));
    *f &= __shfl_xor(*f, d);
  }
}

// A thread takes 8 channels of a token of the keys or the values at a time, the
// D/8 threads of a token beside each other, so a group's are too.  All of a
// thread's loads are on their way before the first is used.
template <int D, int G, bool kOne>
__global__ void __launch_bounds__(kOne ? 64 : 256) kv_append_kernel(KvDev c, int layer, const int32_t* __restrict__ seqs,
                                                             const int32_t* __restrict__ starts,
                                                             const int32_t* __restrict__ cu, int n_tokens,
                                                             int max_new, KvRows k, KvRows v,
                                                             int32_t* __restrict__ d_err) {
  constexpr int CH = D / 8, NG = D / G, kThreads = kOne ? 64 : 256, kItems = kOne ? 1 : 2 * 32 * CH / kThreads;
  const int b = blockIdx.z, h = blockIdx.y;
  const Row r = row_of(c, seqs, starts, cu, b, n_tokens, max_new);
  const bool lead = blockIdx.x == 0 && h == 0 && threadIdx.x == 0;
  if (r.start < 0) return;
  if (r.seq < 0 || r.seq >= c.n_seqs) {
    if (lead && d_err) atomicAdd(d_err, 1);
    return;
  }
  if (blockIdx.x == 0 && h == 0 && d_err) {
    // A row counts once: what it may not write, or has no page for.
    int bad = r.over;
    const int64_t s0 = r.start >> c.page_shift, s1 = r.n > 0 ? ((int64_t)r.start + r.n - 1) >> c.page_shift : s0 - 1;
    for (int64_t s = s0 + threadIdx.x; s <= s1; s += blockDim.x) {
      const int page = s < c.max_pages ? c.pages[(int64_t)r.seq * c.max_pages + s] : -1;
      bad |= page < 0 || page >= c.n_pages;
    }
    bad = __syncthreads_or(bad);
    if (lead && bad) atomicAdd(d_err, 1);
  }
  const int64_t rec = (r.start >> 5) + blockIdx.x;
  const int t0 = (int)max((int64_t)0, r.start - rec * 32);                             // new tokens of the record: [t0, t1)
  const int t1 = (int)min((int64_t)32, (int64_t)r.start + r.n - rec * 32);
  if (t0 >= t1) return;
  uint8_t* out = record(c, layer, r.seq, rec, h);
  if (out == nullptr) return;
  uint32_t* kw = reinterpret_cast<uint32_t*>(out);
  uint32_t* vw = kw + 4 * D;
  uint32_t* params = kw + 8 * D;
  __shared__ uint32_t codes[32][D / 4 + 2];   // the values' codes, a byte each
  const int64_t tok = (int64_t)r.first + rec * 32 - r.start;   // the call's token of the record's token 0
  // Items slot, slot + kThreads / CH, ...: the tokens' keys, then their values.
  const int ch = threadIdx.x % CH, slot = threadIdx.x / CH;
  auto token = [&](int at) { return kOne ? t0 : at & 31; };
  auto is_value = [&](int at) { return kOne ? at > 0 : at >= 32; };
  auto is_new = [&](int at) { return kOne ? at < 2 : token(at) >= t0 && token(at) < t1; };
  half8 x[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const int at = slot + i * (kThreads / CH);
    const half8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
    const KvRows& src = is_value(at) ? v : k;
    x[i] = is_new(at) ? load8(src.p + (tok + token(at)) * src.ts + h * src.hs + ch * 8) : zero;
  }
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const int at = slot + i * (kThreads / CH), t = token(at);
    float lo = (float)x[i][0], hi = lo;
    int f = 1;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float xe = (float)x[i][e];
      lo = fminf(lo, xe);
      hi = fmaxf(hi, xe);
      f &= xe - xe == 0.0f;
    }
    reduce_group<G / 8>(&lo, &hi, &f);
    const Q4Params p = q4_params(lo, hi, f != 0);
    uint32_t q[8];
    q4_codes(x[i], lo, (float)p.s, q);
    if (!is_new(at)) continue;
    if (!is_value(at)) {
      kw[(((t >> 4) * 4 + (ch & 3)) * 16 + (t & 15)) * (D / 32) + (ch >> 2)] = code_word(q);
    } else {
      codes[t][2 * ch] = q[0] | q[1] << 8 | q[2] << 16 | q[3] << 24;
      codes[t][2 * ch + 1] = q[4] | q[5] << 8 | q[6] << 16 | q[7] << 24;
    }
    if (ch % (G / 8) == 0) params[is_value(at) * 32 * NG + (ch / (G / 8)) * 32 + t] = pair_bits(p);
  }
  __syncthreads();
  // Words of four channels and the eight tokens 4 cc + (0..3) and 16 more: bytes
  // to nibbles, then a 4 x 4 transpose.  (Word of channel d: [D/64][cc][ch 16][jd 4].)
  for (int i = threadIdx.x; i < D; i += kThreads) {
    const int jd = i & 3, c4 = (i >> 2) & 3, cc = (i >> 4) & 3, ld = i >> 6;
    const int d4 = ld * 16 + jd * 4 + c4;   // channels 4 d4 ..
    uint32_t mask = 0, two[4];
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const int t = (m >> 1) * 16 + 4 * cc + 2 * (m & 1);
      uint32_t a = 0, b2 = 0;
      if (t >= t0 && t < t1) {
        a = codes[t][d4];
        mask |= 15u << (8 * m);
      }
      if (t + 1 >= t0 && t + 1 < t1) {
        b2 = codes[t + 1][d4];
        mask |= 240u << (8 * m);
      }
      two[m] = a | b2 << 4;
    }
    if (mask == 0) continue;
    const uint32_t lo01 = __builtin_amdgcn_perm(two[1], two[0], 0x05010400u);   // bytes 0, 0', 1, 1'
    const uint32_t hi01 = __builtin_amdgcn_perm(two[1], two[0], 0x07030602u);
    const uint32_t lo23 = __builtin_amdgcn_perm(two[3], two[2], 0x05010400u);
    const uint32_t hi23 = __builtin_amdgcn_perm(two[3], two[2], 0x07030602u);
    uint32_t w[4];
    w[0] = (lo01 & 0xFFFFu) | lo23 << 16;
    w[1] = lo01 >> 16 | (lo23 & 0xFFFF0000u);
    w[2] = (hi01 & 0xFFFFu) | hi23 << 16;
    w[3] = hi01 >> 16 | (hi23 & 0xFFFF0000u);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t* at = vw + ((ld * 4 + cc) * 16 + c4 * 4 + e) * 4 + jd;
      *at = mask == 0xFFFFFFFFu ? w[e] : w[e] | (*at & ~mask);
    }
  }
}

__global__ void __launch_bounds__(256) kv_read_kernel(KvDev c, int layer, const int32_t* __restrict__ seqs,
                                                      const int32_t* __restrict__ starts,
                                                      const int32_t* __restrict__ cu, int n_tokens, int max_new,
                                                      uint16_t* __restrict__ k, uint16_t* __restrict__ v) {
  const int b = blockIdx.z, h = blockIdx.y;
  Row r = row_of(c, seqs, starts, cu, b, n_tokens, max_new);
  const bool none = r.start < 0 || r.seq < 0 || r.seq >= c.n_seqs;
  if (none) r.start = 0;
  const int64_t rec = (r.start >> 5) + blockIdx.x;
  const int t0 = (int)max((int64_t)0, r.start - rec * 32);
  const int t1 = (int)min((int64_t)32, (int64_t)r.start + r.n - rec * 32);
  if (t0 >= t1) return;
  const uint8_t* in = none ? nullptr : record(c, layer, r.seq, rec, h);
  const int CH = c.D >> 3, NG = c.D / c.G;
  const int64_t tok = (int64_t)r.first + rec * 32 - r.start;
  const uint32_t* kw = reinterpret_cast<const uint32_t*>(in);
  const uint32_t* params = kw + 8 * c.D;
  __shared__ uint32_t vw[4 * 256];
  if (in != nullptr)
    for (int i = threadIdx.x; i < 4 * c.D; i += blockDim.x) vw[i] = kw[4 * c.D + i];
  __syncthreads();
  const int items = 2 * (t1 - t0) * CH;
  for (int i = threadIdx.x; i < items; i += blockDim.x) {
    const int ch = i % CH, t = t0 + (i / CH) % (t1 - t0), which = i / (CH * (t1 - t0));
    half8 x = {0, 0, 0, 0, 0, 0, 0, 0};
    if (in != nullptr) {
      const uint32_t p = params[which * 32 * NG + (ch * 8 / c.G) * 32 + t];
      const float s = lo_half(p), m = hi_half(p);
      if (which == 0) {
        const uint32_t w = kw[(((t >> 4) * 4 + (ch & 3)) * 16 + (t & 15)) * (c.D >> 5) + (ch >> 2)];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (_Float16)q4_value((w >> (4 * nibble_of(e))) & 15u, s, m);
      } else {
        const int cc = (t & 15) >> 2, n = (t >> 4) * 4 + (t & 3);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int d = ch * 8 + e;
          const uint32_t w = vw[(((d >> 6) * 4 + cc) * 16 + (d & 15)) * 4 + ((d >> 4) & 3)];
          x[e] = (_Float16)q4_value((w >> (4 * n)) & 15u, s, m);
        }
      }
    }
    uint16_t* o = (which ? v : k) + ((tok + t) * c.H + h) * c.D + ch * 8;
    *reinterpret_cast<half8*>(o) = x;
  }
}

// Records that n tokens from any start touch at most.
int64_t records(int max_new) { return ((int64_t)max_new + 30) / 32 + 1; }

}  // namespace

hipError_t launch_kv_append(const KvDev& c, int layer, const int32_t* seqs, const int32_t* starts,
                            const int32_t* cu, int n_rows, int n_tokens, int max_new, const KvRows& k,
                            const KvRows& v, int32_t* d_err, hipStream_t s) {
  const dim3 grid((uint32_t)records(max_new), c.H, n_rows);
  // A token a row is one wave's work (32 lanes of it at D = 128).
#define TQ_APPEND(D, G)                                                                                            \
  if (max_new == 1)                                                                                                \
    kv_append_kernel<D, G, true><<<grid, 64, 0, s>>>(c, layer, seqs, starts, cu, n_tokens, max_new, k, v, d_err);  \
  else                                                                                                             \
    kv_append_kernel<D, G, false><<<grid, 256, 0, s>>>(c, layer, seqs, starts, cu, n_tokens, max_new, k, v, d_err)
  if (c.D == 64) {
    if (c.G == 32) { TQ_APPEND(64, 32); } else { TQ_APPEND(64, 64); }
  } else if (c.D == 128) {
    if (c.G == 32) { TQ_APPEND(128, 32); } else if (c.G == 64) { TQ_APPEND(128, 64); } else { TQ_APPEND(128, 128); }
  } else {
    if (c.G == 32) { TQ_APPEND(256, 32); } else if (c.G == 64) { TQ_APPEND(256, 64); } else { TQ_APPEND(256, 128); }
  }
#undef TQ_APPEND
  return hipGetLastError();
}

hipError_t launch_kv_read(const KvDev& c, int layer, const int32_t* seqs, const int32_t* starts, const int32_t* cu,
                          int n_rows, int n_tokens, int max_new, uint16_t* k, uint16_t* v, hipStream_t s) {
  const dim3 grid((uint32_t)records(max_new), c.H, n_rows);
  kv_read_kernel<<<grid, 256, 0, s>>>(c, layer, seqs, starts, cu, n_tokens, max_new, k, v);
  return hipGetLastError();
}

}  // namespace tq
