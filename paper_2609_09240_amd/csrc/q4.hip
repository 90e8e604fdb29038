// Products with 4-bit weights and group parameters (gfx950):
//     w[n][k] = m[n][g] + s[n][g] q[n][k],   q in 0..15
//     y[b][n] = sum_g ( s sum_{k in g} q x[b][k]  +  m sum_{k in g} x[b][k] )
//
// One matrix instruction v_mfma_f32_16x16x32_f16 takes 16 rows of W (the
// codes less 8, exact in fp16; the offsets grow by 8 scales) and 16 rows of X over 32 inputs, for one
// activation row as for sixteen: columns past B repeat row B-1 and are
// dropped.  The codes of a group are summed in a chain of their own, and the
// group's scale multiplies the fp32 sums, four per lane, so no weight is
// formed and nothing is rounded below fp32.  The sum of x is one more
// instruction per 32 inputs with ones in place of the codes, shared by the
// row tiles of a wave.

#include "q4_internal.h"

namespace tq {
namespace {

constexpr int kWaves = 8;

__device__ inline float4v mfma(half8 a, half8 b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// ---- Quantise and unpack: a workgroup per tile of 16 rows and 128 inputs, a
// thread per 8 inputs of a row.

__global__ void __launch_bounds__(256) q4_quantize_kernel(const uint16_t* __restrict__ w, int64_t ldw, int N, int K,
                                                          int KB, int G, uint32_t* __restrict__ codes,
                                                          uint32_t* __restrict__ params) {
  const int T = blockIdx.x / KB, blk = blockIdx.x % KB;
  const int r = threadIdx.x >> 4, ch = threadIdx.x & 15;
  const int64_t n = (int64_t)T * 16 + r;
  const int k = blk * 128 + ch * 8;
  float x[8];
  float lo = __builtin_inff(), hi = -__builtin_inff();
  bool finite = true;
  const int have = n < N ? min(8, max(0, K - k)) : 0;
  if (have == 8) {
    const half8 v = load8(w + n * ldw + k);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = e < have ? lo_half(w[n * ldw + k + e]) : 0.0f;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < have) {
      lo = fminf(lo, x[e]);
      hi = fmaxf(hi, x[e]);
      finite = finite && (x[e] - x[e] == 0.0f);
    }
  int f = finite;
  for (int d = 1; d < G / 8; d <<= 1) {
    lo = fminf(lo, __shfl_xor(lo, d));
    hi = fmaxf(hi, __shfl_xor(hi, d));
    f &= __shfl_xor(f, d);
  }
  // Nothing of the group is in the matrix: parameters and codes of 0.
  const bool empty = n >= N || (k & ~(G - 1)) >= K;
  Q4Params p;
  p.s = p.m = (_Float16)0.0f;
  if (!empty) p = q4_params(lo, hi, f != 0);
  uint32_t q[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) q[e] = e < have ? q4_code(x[e], lo, (float)p.s) : 0u;
  const int64_t tile = blockIdx.x;
  codes[tile * 256 + ((ch & 3) * 16 + r) * 4 + (ch >> 2)] = code_word(q);
  if ((ch & (G / 8 - 1)) == 0) {
    const int per = 128 / G;
    params[(((int64_t)T * KB + blk) * per + ch / (G / 8)) * 16 + r] = pair_bits(p);
  }
}

__global__ void __launch_bounds__(256) q4_unpack_kernel(const uint32_t* __restrict__ codes,
                                                        const uint32_t* __restrict__ params, int N, int K, int KB,
                                                        int G, uint16_t* __restrict__ w) {
  const int T = blockIdx.x / KB, blk = blockIdx.x % KB;
  const int r = threadIdx.x >> 4, ch = threadIdx.x & 15;
  const int64_t n = (int64_t)T * 16 + r;
  const int k = blk * 128 + ch * 8;
  const int have = n < N ? min(8, max(0, K - k)) : 0;
  if (have == 0) return;
  const int64_t tile = blockIdx.x;
  const uint32_t c = codes[tile * 256 + ((ch & 3) * 16 + r) * 4 + (ch >> 2)];
  const uint32_t p = params[(((int64_t)T * KB + blk) * (128 / G) + ch / (G / 8)) * 16 + r];
  const float s = lo_half(p), m = hi_half(p);
  half8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (_Float16)q4_value((c >> (4 * nibble_of(e))) & 15u, s, m);
  uint16_t* out = w + n * K + k;
  if (have == 8) {
    reinterpret_cast<half8_u*>(out)->v = v;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < have) {
        const _Float16 x = v[e];   // bit_cast of a vector's element itself takes element 0
        out[e] = __builtin_bit_cast(uint16_t, x);
      }
  }
}

// ---- The product.

// y[b][n] as the sum of x times the weights formed one by one: for outputs
// that are not finite, where the sums over codes are not what the weights
// give (an infinite input times a code of 0).
__device__ __attribute__((noinline)) float by_weights(const uint8_t* codes, const uint16_t* params, int K, int KB,
                                                      int G, const uint16_t* x, int64_t n) {
  const uint32_t* cw = reinterpret_cast<const uint32_t*>(codes);
  const uint32_t* pw = reinterpret_cast<const uint32_t*>(params);
  const int64_t T = n >> 4;
  const int r = (int)(n & 15);
  float acc = 0.0f;
  for (int k = 0; k < K; ++k) {
    const int blk = k >> 7, j = (k >> 5) & 3, c = (k >> 3) & 3, e = k & 7;
    const uint32_t w = cw[((T * KB + blk) * 64 + c * 16 + r) * 4 + j];
    const uint32_t p = pw[(T * KB * (128 / G) + k / G) * 16 + r];
    acc = fmaf(q4_value((w >> (4 * nibble_of(e))) & 15u, lo_half(p), hi_half(p)), lo_half(x[k]), acc);
  }
  return acc;
}

// Inputs 8 from k on, zeros past K.
__device__ inline half8 load_tail(const uint16_t* x, int k, int K) {
  half8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = k + e < K ? __builtin_bit_cast(_Float16, x[k + e]) : (_Float16)0.0f;
  return v;
}

template <int G, int RT, int CT>
struct Block {
  u4v w[RT];
  u4v p[RT][128 / G];
  half8 x[CT][4];
};

template <int G, int RT, int CT>
__global__ void __launch_bounds__(64 * kWaves) q4_gemm_kernel(const uint8_t* __restrict__ codes,
                                                              const uint16_t* __restrict__ params,
                                                              const uint16_t* __restrict__ X, int64_t ldx, int N,
                                                              int K, int B, void* __restrict__ Y, int out_f32) {
  constexpr int NG = 128 / G, J = G / 32;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane >> 4, col = lane & 15;
  const int KB = (K + 127) >> 7, NT = (N + 15) >> 4;
  const int T0 = blockIdx.x * RT;
  const uint16_t* xp[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) xp[ct] = X + (int64_t)min(col + 16 * ct, B - 1) * ldx;
  const u4v* wp[RT];
  const u4v* pp[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int64_t T = min(T0 + rt, NT - 1);
    wp[rt] = reinterpret_cast<const u4v*>(codes + T * KB * 1024) + lane;
    pp[rt] = reinterpret_cast<const u4v*>(params + T * KB * NG * 32) + c;
  }
  const half8 ones = {(_Float16)1, (_Float16)1, (_Float16)1, (_Float16)1,
                      (_Float16)1, (_Float16)1, (_Float16)1, (_Float16)1};
  float4v acc[RT][CT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) acc[rt][ct] = float4v{0, 0, 0, 0};

  typedef Block<G, RT, CT> Blk;
  auto load = [&](Blk& d, int blk) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      d.w[rt] = wp[rt][(int64_t)blk * 64];
#pragma unroll
      for (int g = 0; g < NG; ++g) d.p[rt][g] = pp[rt][(int64_t)(blk * NG + g) * 4];
    }
    if (blk * 128 + 128 <= K) {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int j = 0; j < 4; ++j) d.x[ct][j] = load8(xp[ct] + blk * 128 + 32 * j + 8 * c);
    } else {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int j = 0; j < 4; ++j) d.x[ct][j] = load_tail(xp[ct], blk * 128 + 32 * j + 8 * c, K);
    }
  };
  auto compute = [&](const Blk& d) {
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      float xs[CT];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        float4v t = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < J; ++j) t = mfma(ones, d.x[ct][g * J + j], t);
        xs[ct] = t[0];
      }
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        half8 a[J];
#pragma unroll
        for (int j = 0; j < J; ++j) a[j] = code_operand(d.w[rt][g * J + j]);
        float s[4], m[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          m[i] = centred(lo_half(d.p[rt][g][i]), hi_half(d.p[rt][g][i]));
          s[i] = lo_half(d.p[rt][g][i]) * kCodeUnit;
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          float4v t = {0, 0, 0, 0};
#pragma unroll
          for (int j = 0; j < J; ++j) t = mfma(a[j], d.x[ct][g * J + j], t);
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[rt][ct][i] = fmaf(s[i], t[i], fmaf(m[i], xs[ct], acc[rt][ct][i]));
        }
      }
    }
  };

  if constexpr (CT == 4) {   // four column tiles leave no registers for the next block
    for (int blk = wave; blk < KB; blk += kWaves) {
      Blk cur;
      load(cur, blk);
      compute(cur);
    }
  } else {
  Blk cur, nxt;
  if (wave < KB) load(cur, wave);
  for (int blk = wave; blk < KB; blk += kWaves) {
    const bool more = blk + kWaves < KB;
    if (more) load(nxt, blk + kWaves);
    compute(cur);
    if (more) cur = nxt;
  }
  }

  // The waves' sums, added in the waves' order.
  __shared__ float4v part[kWaves][RT * CT][64];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) part[wave][rt * CT + ct][lane] = acc[rt][ct];
  __syncthreads();
  for (int i = threadIdx.x; i < RT * CT * 64; i += 64 * kWaves) {
    const int l = i & 63, ct = (i >> 6) % CT, rt = (i >> 6) / CT;
    const int b = 16 * ct + (l & 15);
    const int64_t n = (int64_t)(T0 + rt) * 16 + 4 * (l >> 4);
    if (b >= B || n >= N) continue;
    float4v y = part[0][rt * CT + ct][l];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) y += part[w][rt * CT + ct][l];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (n + e >= N) break;
      float v = y[e];
      if (!(fabsf(v) < __builtin_inff())) v = by_weights(codes, params, K, KB, G, X + (int64_t)b * ldx, n + e);
      const int64_t at = (int64_t)b * N + n + e;
      if (out_f32)
        static_cast<float*>(Y)[at] = v;
      else
        static_cast<_Float16*>(Y)[at] = (_Float16)v;
    }
  }
}

template <int G, int RT, int CT>
void start(const Q4Dev& m, const uint16_t* X, int64_t ldx, int B, void* Y, bool out_f32, hipStream_t s) {
  const int NT = (m.n_out + 15) / 16;
  q4_gemm_kernel<G, RT, CT><<<(NT + RT - 1) / RT, 64 * kWaves, 0, s>>>(m.codes, m.params, X, ldx, m.n_out, m.n_in, B, Y,
                                                                     out_f32 ? 1 : 0);
}

template <int G>
void start_g(const Q4Dev& m, const uint16_t* X, int64_t ldx, int B, void* Y, bool out_f32, hipStream_t s) {
  const int NT = (m.n_out + 15) / 16;
  if (B <= 16) {
    if (NT >= 2048)
      start<G, G == 32 ? 2 : 4, 1>(m, X, ldx, B, Y, out_f32, s);
    else
      start<G, 1, 1>(m, X, ldx, B, Y, out_f32, s);
  } else if (B <= 32) {
    start<G, 1, 2>(m, X, ldx, B, Y, out_f32, s);
  } else {
    start<G, 1, 4>(m, X, ldx, B, Y, out_f32, s);
  }
}

}  // namespace

hipError_t launch_q4_quantize(const uint16_t* w, int64_t ldw, const Q4Dev& m, uint8_t* codes, uint16_t* params,
                              hipStream_t s) {
  const int NT = (m.n_out + 15) / 16, KB = (m.n_in + 127) / 128;
  q4_quantize_kernel<<<(uint32_t)((int64_t)NT * KB), 256, 0, s>>>(w, ldw, m.n_out, m.n_in, KB, m.group,
                                                                 reinterpret_cast<uint32_t*>(codes),
                                                                 reinterpret_cast<uint32_t*>(params));
  return hipGetLastError();
}

hipError_t launch_q4_unpack(const Q4Dev& m, uint16_t* w, hipStream_t s) {
  const int NT = (m.n_out + 15) / 16, KB = (m.n_in + 127) / 128;
  q4_unpack_kernel<<<(uint32_t)((int64_t)NT * KB), 256, 0, s>>>(reinterpret_cast<const uint32_t*>(m.codes),
                                                               reinterpret_cast<const uint32_t*>(m.params), m.n_out,
                                                               m.n_in, KB, m.group, w);
  return hipGetLastError();
}

hipError_t launch_q4_gemm(const Q4Dev& m, const uint16_t* X, int64_t ldx, int B, void* Y, bool out_f32,
                          hipStream_t s) {
  if (m.group == 32)
    start_g<32>(m, X, ldx, B, Y, out_f32, s);
  else if (m.group == 64)
    start_g<64>(m, X, ldx, B, Y, out_f32, s);
  else
    start_g<128>(m, X, ldx, B, Y, out_f32, s);
  return hipGetLastError();
}

}  // namespace tq
