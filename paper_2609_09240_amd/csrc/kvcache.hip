// Writing and reading the 4-bit key/value cache (gfx950).
//
// A workgroup owns one record: 32 tokens of one head of one row of the call.
// Keys go to their words straight from the thread that quantised them (8
// channels of a token are one word); values cross over LDS, because a word
// of theirs holds 8 tokens of one channel.  A word that also holds tokens
// that are not new is read, changed and written back by one thread.

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

__global__ void kv_append_kernel(KvDev c, int layer, const int32_t* __restrict__ seqs,
                                 const int32_t* __restrict__ starts, const int32_t* __restrict__ cu, int n_tokens,
                                 int max_new, KvRows k, KvRows v, int32_t* __restrict__ d_err) {
  const int b = blockIdx.z, h = blockIdx.y;
  const Row r = row_of(c, seqs, starts, cu, b, n_tokens, max_new);
  const bool lead = blockIdx.x == 0 && h == 0 && threadIdx.x == 0;
  if (r.start < 0) return;
  if (r.seq < 0 || r.seq >= c.n_seqs) {
    if (lead && d_err) atomicAdd(d_err, 1);
    return;
  }
  if (lead && d_err) {
    // A row counts once: what it may not write, or has no page for.
    bool bad = r.over;
    for (int64_t s = r.start >> c.page_shift; !bad && r.n > 0 && s <= ((int64_t)r.start + r.n - 1) >> c.page_shift; ++s) {
      const int page = s < c.max_pages ? c.pages[(int64_t)r.seq * c.max_pages + s] : -1;
      bad = page < 0 || page >= c.n_pages;
    }
    if (bad) atomicAdd(d_err, 1);
  }
  const int64_t rec = (r.start >> 5) + blockIdx.x;
  const int t0 = (int)max((int64_t)0, r.start - rec * 32);                             // new tokens of the record: [t0, t1)
  const int t1 = (int)min((int64_t)32, (int64_t)r.start + r.n - rec * 32);
  if (t0 >= t1) return;
  uint8_t* out = record(c, layer, r.seq, rec, h);
  if (out == nullptr) return;
  uint32_t* kw = reinterpret_cast<uint32_t*>(out);
  uint32_t* vw = kw + 4 * c.D;
  uint32_t* params = kw + 8 * c.D;
  __shared__ uint8_t codes[32][256 + 4];
  const int CH = c.D >> 3, per = c.G >> 3, NG = c.D / c.G;
  const int64_t tok = (int64_t)r.first + rec * 32 - r.start;   // the call's token of the record's token 0
  // A thread takes 8 channels of a token of the keys or the values; the D/8
  // threads of a token are neighbours, so a group's threads are too.
  const int items = 2 * (t1 - t0) * CH;
  for (int i = threadIdx.x; i - (int)threadIdx.x < items; i += blockDim.x) {
    const bool in = i < items;
    const int ii = in ? i : 0;
    const int ch = ii % CH, t = t0 + (ii / CH) % (t1 - t0), which = ii / (CH * (t1 - t0));
    const KvRows& src = which ? v : k;
    const half8 x = load8(src.p + (tok + t) * src.ts + h * src.hs + ch * 8);
    float lo = __builtin_inff(), hi = -__builtin_inff();
    int f = 1;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float xe = (float)x[e];
      lo = fminf(lo, xe);
      hi = fmaxf(hi, xe);
      f &= xe - xe == 0.0f;
    }
    for (int d = 1; d < per; d <<= 1) {
      lo = fminf(lo, __shfl_xor(lo, d));
      hi = fmaxf(hi, __shfl_xor(hi, d));
      f &= __shfl_xor(f, d);
    }
    const Q4Params p = q4_params(lo, hi, f != 0);
    uint32_t q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = q4_code((float)x[e], lo, (float)p.s);
    if (!in) continue;
    if (which == 0) {
      kw[(((t >> 4) * 4 + (ch & 3)) * 16 + (t & 15)) * (c.D >> 5) + (ch >> 2)] = code_word(q);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) codes[t][ch * 8 + e] = (uint8_t)q[e];
    }
    if (ch % per == 0) params[which * 32 * NG + (ch / per) * 32 + t] = pair_bits(p);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 4 * c.D; i += blockDim.x) {
    // word i: [D/64][c 4][ch 16][jd 4]
    const int d = (i >> 8) * 64 + (i & 3) * 16 + ((i >> 2) & 15), cc = (i >> 6) & 3;
    uint32_t w = 0, mask = 0;
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      const int t = (n >> 2) * 16 + 4 * cc + (n & 3);
      if (t >= t0 && t < t1) {
        w |= (uint32_t)codes[t][d] << (4 * n);
        mask |= 15u << (4 * n);
      }
    }
    if (mask == 0) continue;
    if (mask != 0xFFFFFFFFu) w |= vw[i] & ~mask;
    vw[i] = w;
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
  kv_append_kernel<<<grid, 256, 0, s>>>(c, layer, seqs, starts, cu, n_tokens, max_new, k, v, d_err);
  return hipGetLastError();
}

hipError_t launch_kv_read(const KvDev& c, int layer, const int32_t* seqs, const int32_t* starts, const int32_t* cu,
                          int n_rows, int n_tokens, int max_new, uint16_t* k, uint16_t* v, hipStream_t s) {
  const dim3 grid((uint32_t)records(max_new), c.H, n_rows);
  kv_read_kernel<<<grid, 256, 0, s>>>(c, layer, seqs, starts, cu, n_tokens, max_new, k, v);
  return hipGetLastError();
}

}  // namespace tq
