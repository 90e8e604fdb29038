// What the 4-bit operators share: their device-side views, launchers and the
// words of eight codes.  Every launcher assumes its arguments were checked
// on the host (q4_api.hip) and returns the status of the launch.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/tq.h"

namespace tq {

// ---- Matrices (q4.hip).
struct Q4Dev {
  const uint8_t* codes;
  const uint16_t* params;
  int32_t n_out, n_in, group;
};

hipError_t launch_q4_quantize(const uint16_t* w, int64_t ldw, const Q4Dev& m, uint8_t* codes, uint16_t* params,
                              hipStream_t s);
hipError_t launch_q4_unpack(const Q4Dev& m, uint16_t* w, hipStream_t s);
size_t q4_workspace_bytes(const Q4Dev& m, int B);
hipError_t launch_q4_gemm(const Q4Dev& m, const uint16_t* X, int64_t ldx, int B, void* Y, bool out_f32, void* ws,
                          hipStream_t s);

// ---- Cache (kvcache.hip, kvpages.hip, kvattn.hip).
__host__ __device__ inline int64_t kv_record_bytes(int D, int G) { return 32 * (int64_t)(D + 8 * D / G); }

struct KvDev {
  uint8_t* data;
  int32_t* pages;
  int32_t* lens;
  int32_t* refs;
  int64_t page_bytes;
  int64_t layer_bytes;   // n_pages * page_bytes
  int32_t n_layers, H, D, G, page_size, page_shift, n_seqs, max_pages, n_pages;
};

struct KvRows {
  const uint16_t* p;
  int64_t ts, hs;
};

hipError_t launch_kv_append(const KvDev& c, int layer, const int32_t* seqs, const int32_t* starts,
                            const int32_t* cu, int n_rows, int n_tokens, int max_new, const KvRows& k,
                            const KvRows& v, int32_t* d_err, hipStream_t s);
hipError_t launch_kv_read(const KvDev& c, int layer, const int32_t* seqs, const int32_t* starts, const int32_t* cu,
                          int n_rows, int n_tokens, int max_new, uint16_t* k, uint16_t* v, hipStream_t s);

hipError_t launch_kv_extend(const KvDev& c, const int32_t* seqs, const int32_t* cu, int n_rows, int32_t* starts,
                            int32_t* d_err, hipStream_t s);
hipError_t launch_kv_free(const KvDev& c, const int32_t* seqs, int n_rows, int32_t* d_err, hipStream_t s);
size_t kv_workspace_bytes(const KvDev& c, int n_rows);
hipError_t launch_kv_fork(const KvDev& c, const int32_t* parents, const int32_t* children, int n_rows,
                          int32_t* d_err, void* ws, hipStream_t s);
hipError_t launch_kv_compact(const KvDev& c, int32_t* n_live, void* ws, hipStream_t s);
hipError_t launch_kv_copy_pages(const KvDev& c, const int32_t* src, const int32_t* dst, int n, int32_t* d_err,
                                hipStream_t s);

struct AttnCall {
  int32_t n_rows, n_tokens, max_q, n_heads, max_len, window;
  float scale;
  bool out_f32;
  const int32_t* seqs;
  const int32_t* cu;
  KvRows q;
  void* o;
  float* lse;
  void* ws;
};
// false where the launch would not fit a grid.
bool kv_attention_plan(const KvDev& c, const AttnCall& a, size_t* ws_bytes);
hipError_t launch_kv_attention(const KvDev& c, int layer, const AttnCall& a, hipStream_t s);


typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t u4v __attribute__((ext_vector_type(4)));
typedef uint32_t u2v __attribute__((ext_vector_type(2)));

// Eight fp16 values from anywhere (2-byte aligned): one 16-byte load, which
// the hardware takes at any address.
struct __attribute__((packed, aligned(2))) half8_u {
  half8 v;
};
__device__ inline half8 load8(const uint16_t* p) { return reinterpret_cast<const half8_u*>(p)->v; }

// A word of eight codes as an operand of a matrix instruction: code n as the
// fp16 number (n - 8) * 2^-9, register r the nibbles r and r + 4.  The bits of
// a code, masked, are the subnormal number n * 2^-24 (n * 2^-20 where they sit
// 4 bits up); one exact multiply-add makes it normal and centred: 9
// instructions for 8 codes, and kCodeUnit is left to the fp32 sums.
// Around 0, which costs nothing: cached values are summed so, with offset +
// 8 scale in the place of the offset, and both sums are small where the values
// are; products and keys start the sum of their codes at 8 times that of the
// other operand, and multiply the offset as it is.
// Normal, because the matrix cores align products by their operands' exponents
// alone: subnormal codes, which would save the multiply-add, lose 7 bits of the
// sum (measured: 7.6e-6 off where a product is now 1.3e-7 off).  The other
// operand may be subnormal: its bits lie within ten below 2^-14, and with four
// of a code that is less than the sum holds (measured: 1e-7 off or less).
constexpr float kCodeUnit = 512.0f;
__device__ inline half8 code_operand(uint32_t w) {
  const half2v a = {(_Float16)32768.0f, (_Float16)32768.0f}, b = {(_Float16)2048.0f, (_Float16)2048.0f};
  const half2v m = {(_Float16)-0.015625f, (_Float16)-0.015625f};
  const uint32_t t = w >> 8;
  const half2v r0 = __builtin_elementwise_fma(__builtin_bit_cast(half2v, w & 0x000F000Fu), a, m);
  const half2v r1 = __builtin_elementwise_fma(__builtin_bit_cast(half2v, w & 0x00F000F0u), b, m);
  const half2v r2 = __builtin_elementwise_fma(__builtin_bit_cast(half2v, t & 0x000F000Fu), a, m);
  const half2v r3 = __builtin_elementwise_fma(__builtin_bit_cast(half2v, t & 0x00F000F0u), b, m);
  return half8{r0[0], r0[1], r1[0], r1[1], r2[0], r2[1], r3[0], r3[1]};
}
// What crosses workgroups is stored and loaded at device scope, past the
// caches of a die (sc1), so that no cache has to be written back or
// invalidated: fences around the count of a join cost attention 200 us a call,
// these 2.
constexpr int kCoherent = 16;
__device__ __forceinline__ void put4(__amdgpu_buffer_rsrc_t r, int at, float4v v) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4v, v), r, at, 0, kCoherent);
}
__device__ __forceinline__ float4v get4(__amdgpu_buffer_rsrc_t r, int at) {
  return __builtin_bit_cast(float4v, __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, kCoherent));
}

// Inclusive prefix sum over a wave.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);   // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);   // row_bcast 15 to rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);   // row_bcast 31 to rows 2 and 3
  return x;
}

// Lane n of each 16 to all of them (n a constant).
#define TQ_ROW_BCAST(n) case n: return __builtin_amdgcn_update_dpp(0, x, 0x150 + n, 0xF, 0xF, false);
__device__ __forceinline__ uint32_t row_bcast(uint32_t x, int n) {
  switch (n) {
    TQ_ROW_BCAST(0) TQ_ROW_BCAST(1) TQ_ROW_BCAST(2) TQ_ROW_BCAST(3) TQ_ROW_BCAST(4) TQ_ROW_BCAST(5)
    TQ_ROW_BCAST(6) TQ_ROW_BCAST(7) TQ_ROW_BCAST(8) TQ_ROW_BCAST(9) TQ_ROW_BCAST(10) TQ_ROW_BCAST(11)
    TQ_ROW_BCAST(12) TQ_ROW_BCAST(13) TQ_ROW_BCAST(14)
    default: return __builtin_amdgcn_update_dpp(0, x, 0x15F, 0xF, 0xF, false);
  }
}
#undef TQ_ROW_BCAST

// Nibble of element e of eight, and eight codes as a word.
__device__ inline constexpr int nibble_of(int e) { return (e & 1) * 4 + (e >> 1); }
__device__ inline uint32_t code_word(const uint32_t* q) {
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) w |= q[e] << (4 * nibble_of(e));
  return w;
}

// The quantiser's arithmetic for one group: scale and offset from the
// smallest and largest value, and a code.
struct Q4Params {
  _Float16 s, m;
};
__device__ inline Q4Params q4_params(float lo, float hi, bool finite) {
  Q4Params p;
  p.m = (_Float16)lo;
  p.s = (_Float16)__fdiv_rn(__fsub_rn(hi, lo), 15.0f);
  if (!finite) p.s = p.m = (_Float16)__builtin_nanf("");
  return p;
}
// Codes of eight values of a group.  The quotient by a reciprocal is within
// 2^-18 of the rounded one; where it lies further than that from a half both
// round to the same code, and only elsewhere is the division made.
__device__ __forceinline__ void q4_codes(half8 x, float lo, float s, uint32_t (&q)[8]) {
  const float inv = 1.0f / s;
  float d[8], t[8];
  bool near = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    d[e] = __fsub_rn((float)x[e], lo);
    t[e] = d[e] * inv;
    near |= fabsf(t[e] - floorf(t[e]) - 0.5f) < 3.0e-5f;
  }
  if (!(s > 0.0f)) {   // 0 or NaN
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = 0;
    return;
  }
  if (near || !(inv < __builtin_inff())) {
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = __fdiv_rn(d[e], s);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) q[e] = (uint32_t)fminf(fmaxf(rintf(t[e]), 0.0f), 15.0f);
}
__device__ inline float q4_value(uint32_t q, float s, float m) { return fmaf((float)q, s, m); }

__device__ inline uint32_t pair_bits(Q4Params p) {
  return (uint32_t)__builtin_bit_cast(uint16_t, p.s) | ((uint32_t)__builtin_bit_cast(uint16_t, p.m) << 16);
}
__device__ inline float lo_half(uint32_t b) { return (float)__builtin_bit_cast(_Float16, (uint16_t)b); }
__device__ inline float hi_half(uint32_t b) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(b >> 16)); }

}  // namespace tq
