// Products with 4-bit weights and group parameters (gfx950):
//     w[n][k] = m[n][g] + s[n][g] q[n][k],   q in 0..15
//     y[b][n] = sum_g ( s sum_{k in g} q x[b][k]  +  m sum_{k in g} x[b][k] )
//
// One matrix instruction v_mfma_f32_16x16x32_f16 takes 16 rows of W (the
// codes less 8, exact in fp16) and 16 rows of X over 32 inputs, for one
// activation row as for sixteen: columns past B repeat row B-1 and are
// dropped.  The codes of a group are summed in a chain of their own, which
// starts at 8 times the group's sum of x, and the group's scale and offset
// multiply fp32 sums, four per lane, so no weight is formed and nothing is
// rounded below fp32.  The sum of x is one more instruction per 32 inputs with
// constants in place of the codes, shared by the row tiles of a wave.
//
// Two kernels.  With few rows of X every wave streams blocks of 128 inputs of
// its row tiles straight into registers and reads X as operands from the
// caches; a load of X then touches a line per row, and from 5 rows on (3 where
// there are many row tiles) that costs more than staging X in LDS, which the
// other kernel does.  Kernel times, weights from HBM, groups of 128:
//   1024 x 4096     B = 1 4.0 us (launch and two trips to memory), 64 12.4
//   4096 x 4096     B = 1 4.6, 32 9.7, 64 14.4
//   4096 x 12288    B = 1 8.8, 3 8.9, 8 11.0, 16 11.6, 32 14.7, 64 25.2
//   12288 x 4096    B = 1 8.6, 4 9.7, 16 10.2, 32 14.3, 64 25.9
//   131072 x 4096   B = 1 52.7 (groups of 64: 302 MB, 5.7 TB/s), 16 76
// B = 1 of a large matrix is bound by HBM, of a small one by latency; from B =
// 16 on by X, which every workgroup reads: a workgroup of four row tiles at B =
// 64, or of one at B = 16, brings four times the bytes of X that it brings of
// codes (4096 x 12288: 135 and 127 MB from L2, counted, for 27 of weights).  From
// B = 17 on, where there are few row groups, each is split along K, and the parts
// are joined by the last of them to finish.

#include <atomic>

#include "q4_internal.h"

namespace tq {
namespace {

__device__ inline float4v mfma(half8 a, half8 b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Inputs 8 from k on, zeros past K.
__device__ inline half8 load_tail(const uint16_t* x, int k, int K) {
  half8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = k + e < K ? __builtin_bit_cast(_Float16, x[k + e]) : (_Float16)0.0f;
  return v;
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
  const int have = n < N ? min(8, max(0, K - k)) : 0;
  half8 x = {0, 0, 0, 0, 0, 0, 0, 0};
  if (have == 8)
    x = load8(w + n * ldw + k);
  else if (have > 0)
    x = load_tail(w + n * ldw, k, K);
  float lo = __builtin_inff(), hi = -__builtin_inff();
  int f = 1;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < have) {
      const float v = (float)x[e];
      lo = fminf(lo, v);
      hi = fmaxf(hi, v);
      f &= v - v == 0.0f;
    }
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
  q4_codes(x, lo, (float)p.s, q);
#pragma unroll
  for (int e = 0; e < 8; ++e) q[e] = e < have ? q[e] : 0u;
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
__device__ __attribute__((noinline)) float by_weights(const uint8_t* codes, const uint32_t* pw, int K, int KB,
                                                      int G, const uint16_t* x, int64_t n) {
  const uint32_t* cw = reinterpret_cast<const uint32_t*>(codes);
  const int64_t T = n >> 4;
  const int r = (int)(n & 15);
  float acc = 0.0f;
  for (int k = 0; k < K && acc == acc; k += 8) {   // NaN stays
    const int blk = k >> 7, j = (k >> 5) & 3, c = (k >> 3) & 3;
    const uint32_t w = cw[((T * KB + blk) * 64 + c * 16 + r) * 4 + j];
    const uint32_t p = pw[(T * KB * (128 / G) + k / G) * 16 + r];
    const half8 v = load_tail(x, k, K);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (k + e < K) acc = fmaf(q4_value((w >> (4 * nibble_of(e))) & 15u, lo_half(p), hi_half(p)), (float)v[e], acc);
  }
  return acc;
}

// The parameters of a row tile and block are one word a lane: lane (c, k) holds
// row 4 c + k % 4 of group k / 4, and a broadcast within 16 lanes brings each to
// the lanes whose sums it scales.
template <int NG>
__device__ inline const uint32_t* param_lane(const uint32_t* params, int64_t T, int KB) {
  const int c = (threadIdx.x >> 4) & 3, k = threadIdx.x & 15;
  return params + T * KB * NG * 16 + (k / 4 % NG) * 16 + 4 * c + (k & 3);
}

// One block of 128 inputs of RT row tiles times CT tiles of 16 rows of X, added
// to acc, in the codes' unit.  done(rt) is called once the registers of row
// tile rt's weights are free, for the loads that come next.
template <int G, int RT, int CT, class F>
__device__ __forceinline__ void block_product(const u4v (&w)[RT], const uint32_t (&p)[RT], const half8 (&x)[CT][4],
                                              float4v (&acc)[RT][CT], F done) {
  constexpr int NG = 128 / G, J = G / 32;
  // 8 in the codes' unit: its product with x is the sum of x that codes less 8
  // lack, in all four rows of a lane.
  const _Float16 e8 = (_Float16)(8.0f / kCodeUnit);
  const half8 eights = {e8, e8, e8, e8, e8, e8, e8, e8};
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    float4v z[CT];
    float xs[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      z[ct] = float4v{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < J; ++j) z[ct] = mfma(eights, x[ct][g * J + j], z[ct]);
      xs[ct] = z[ct][0] * 0.125f;   // the sum of x in the codes' unit
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      half8 a[J];
#pragma unroll
      for (int j = 0; j < J; ++j) a[j] = code_operand(w[rt][g * J + j]);
      half2v sm[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) sm[i] = __builtin_bit_cast(half2v, row_bcast(p[rt], 4 * g + i));
      if (g == NG - 1) done(rt);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        float4v t = z[ct];
#pragma unroll
        for (int j = 0; j < J; ++j) t = mfma(a[j], x[ct][g * J + j], t);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          acc[rt][ct][i] = fmaf((float)sm[i][0], t[i], acc[rt][ct][i]);
          acc[rt][ct][i] = fmaf((float)sm[i][1], xs[ct], acc[rt][ct][i]);
        }
      }
    }
  }
}

// Four outputs of a lane: rows 4 (l / 16) + (0..3) of set `set` (its first row
// 16 (T0 + set)), row l % 16 of X's tile ct.
struct Out {
  const uint8_t* codes;
  const uint32_t* params;
  const uint16_t* X;
  int64_t ldx;
  void* Y;
  int N, K, B, G, T0, out_f32;
};
__device__ inline void write_four(const Out& o, int set, int ct, int l, float4v y) {
  const int b = 16 * ct + (l & 15);
  const int64_t n = (int64_t)(o.T0 + set) * 16 + 4 * (l >> 4);
  if (b >= o.B) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (n + e >= o.N) break;
    float v = y[e];
    if (!(fabsf(v) < __builtin_inff()))
      v = by_weights(o.codes, o.params, o.K, (o.K + 127) >> 7, o.G, o.X + (int64_t)b * o.ldx, n + e);
    const int64_t at = (int64_t)b * o.N + n + e;
    if (o.out_f32)
      static_cast<float*>(o.Y)[at] = v;
    else
      static_cast<_Float16*>(o.Y)[at] = (_Float16)v;
  }
}

// The sum over W waves, in their order, of four outputs.
template <int W, int S>
__device__ inline float4v sum_waves(const float4v (*part)[S][64], int i, int l) {
  float4v y = part[0][i][l];
#pragma unroll
  for (int k = 1; k < W; ++k) y += part[k][i][l];
  return y;
}

// Few rows of X: every wave reads the inputs of its block from memory in the
// shape of the operand (16 bytes of up to four rows, 64 bytes apart from each
// other's lanes).  A wave takes the blocks wave, wave + W, ... of RT row tiles;
// the next one is on its way as registers become free.
template <int G, int RT, int W>
__global__ void __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(2))) q4_gemv_kernel(const uint8_t* __restrict__ codes,
                                                         const uint32_t* __restrict__ params,
                                                         const uint16_t* __restrict__ X, int64_t ldx, int N, int K,
                                                         int B, void* __restrict__ Y, int out_f32) {
  constexpr int NG = 128 / G;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane >> 4, col = lane & 15;
  const int KB = (K + 127) >> 7, NT = (N + 15) >> 4;
  const int T0 = blockIdx.x * RT;
  const uint16_t* xp = X + (int64_t)min(col, B - 1) * ldx;
  const u4v* wp[RT];
  const uint32_t* pp[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int64_t T = min(T0 + rt, NT - 1);
    wp[rt] = reinterpret_cast<const u4v*>(codes + T * KB * 1024) + lane;
    pp[rt] = param_lane<NG>(params, T, KB);
  }
  float4v acc[RT][1];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) acc[rt][0] = float4v{0, 0, 0, 0};

  u4v w[RT];
  uint32_t p[RT];
  half8 x[1][4];
  auto load_w = [&](int rt, int blk) {
    w[rt] = wp[rt][(int64_t)blk * 64];
    p[rt] = pp[rt][(int64_t)blk * NG * 16];
  };
  auto load_x = [&](int blk) {
    if (blk * 128 + 128 <= K) {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[0][j] = load8(xp + blk * 128 + 32 * j + 8 * c);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[0][j] = load_tail(xp, blk * 128 + 32 * j + 8 * c, K);
    }
  };
  // Past the last block the last is read again and not used.
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) load_w(rt, min(wave, KB - 1));
  load_x(min(wave, KB - 1));
  for (int blk = wave; blk < KB; blk += W) {
    const int next = min(blk + W, KB - 1);
    // (As a loop of one pass: without it the compiler takes 169 registers where it
    // took 167, and a SIMD holds two waves in place of three.  131072 x 4096 at B =
    // 1, groups of 64: 58.9 us and 53.5.)
#pragma unroll
    for (int once = 0; once < 1; ++once) {
      block_product<G, RT, 1>(w, p, x, acc, [&](int rt) { load_w(rt, next); });
      load_x(next);
    }
  }
  __shared__ float4v part[W][RT][64];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) part[wave][rt][lane] = acc[rt][0] * kCodeUnit;
  __syncthreads();
  const Out o = {codes, params, X, ldx, Y, N, K, B, G, T0, out_f32};
  for (int i = threadIdx.x; i < RT * 64; i += 64 * W)
    write_four(o, i >> 6, 0, i & 63, sum_waves<W, RT>(part, i >> 6, i & 63));
}

// More rows of X: chunks of 128 WK inputs of all rows go through LDS, whole
// lines of X from memory and operands from LDS, one chunk computed while the
// next arrives.  Wave wr WK + wk takes block wk of a chunk and the row tiles
// RT wr ..  of the workgroup's RT WR.  Where gridDim.y > 1 a workgroup has a part
// of the chunks; the last of a row group's workgroups to finish adds the parts
// in their order and sets the group's count back to 0.
template <int G, int CT, int WK, int WR, int RT>
__global__ void __launch_bounds__(64 * WK * WR) q4_gemm_kernel(const uint8_t* __restrict__ codes,
                                                               const uint32_t* __restrict__ params,
                                                               const uint16_t* __restrict__ X, int64_t ldx, int N,
                                                               int K, int B, void* __restrict__ Y, int out_f32,
                                                               int32_t* __restrict__ count, float* __restrict__ parts) {
  constexpr int NG = 128 / G, KC = 128 * WK, kThreads = 64 * WK * WR, kRow = KC + 8;   // 16 bytes between rows: all banks
  constexpr int kLoads = 16 * CT * (KC / 8) / kThreads, S = WR * RT * CT;
  extern __shared__ __align__(16) uint16_t lds[];   // [2][16 CT][kRow], then the waves' sums over it
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wk = wave % WK, wr = wave / WK;
  const int c = lane >> 4, col = lane & 15;
  const int KB = (K + 127) >> 7, NT = (N + 15) >> 4, all = (KB + WK - 1) / WK;
  const int first = (int)((int64_t)all * blockIdx.y / gridDim.y), chunks = (int)((int64_t)all * (blockIdx.y + 1) / gridDim.y);
  const int T0 = blockIdx.x * WR * RT;
  const u4v* wp[RT];
  const uint32_t* pp[RT];
  float4v acc[RT][CT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int64_t T = min(T0 + wr * RT + rt, NT - 1);
    wp[rt] = reinterpret_cast<const u4v*>(codes + T * KB * 1024) + lane;
    pp[rt] = param_lane<NG>(params, T, KB);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) acc[rt][ct] = float4v{0, 0, 0, 0};
  }

  // Thread i of the workgroup brings 8 inputs of kLoads rows, of two chunks in
  // turn.
  half8 in[2][kLoads];
  auto fetch = [&](int s, int chunk) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = threadIdx.x + i * kThreads, row = at / (KC / 8), k = chunk * KC + at % (KC / 8) * 8;
      const uint16_t* xr = X + (int64_t)min(row, B - 1) * ldx;
      if (k + 8 <= K)
        in[s][i] = load8(xr + k);
      else
        in[s][i] = load_tail(xr, k, K);
    }
  };
  auto stage = [&](int s, int buf) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = threadIdx.x + i * kThreads, row = at / (KC / 8);
      *reinterpret_cast<half8*>(&lds[(buf * 16 * CT + row) * kRow + at % (KC / 8) * 8]) = in[s][i];
    }
  };
  u4v w[2][RT];
  uint32_t p[2][RT];
  auto load_w = [&](int s, int rt, int chunk) {
    const int blk = min(chunk * WK + wk, KB - 1);
    w[s][rt] = wp[rt][(int64_t)blk * 64];
    p[s][rt] = pp[rt][(int64_t)blk * NG * 16];
  };
  if (first < chunks) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) load_w(0, rt, first);
    fetch(0, first);
    if (first + 1 < chunks) fetch(1, first + 1);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) load_w(1, rt, first + 1);
    stage(0, 0);
  }
  __syncthreads();
  for (int chunk0 = first; chunk0 < chunks; chunk0 += 2) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int chunk = chunk0 + s;
      if (chunk >= chunks) break;
      const bool more = chunk + 1 < chunks;
      if (chunk + 2 < chunks) fetch(s, chunk + 2);
      half8 x[CT][4];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          x[ct][j] = *reinterpret_cast<const half8*>(&lds[(s * 16 * CT + 16 * ct + col) * kRow + wk * 128 + 32 * j + 8 * c]);
      // Blocks past the last one meet inputs of 0 only.
      block_product<G, RT, CT>(w[s], p[s], x, acc, [&](int rt) { load_w(s, rt, chunk + 2); });
      if (more) stage(s ^ 1, s ^ 1);
      __syncthreads();
    }
  }
  typedef float4v Part[S][64];
  Part* part = reinterpret_cast<Part*>(lds);
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) part[wk][(wr * RT + rt) * CT + ct][lane] = acc[rt][ct] * kCodeUnit;
  __syncthreads();
  const Out o = {codes, params, X, ldx, Y, N, K, B, G, T0, out_f32};
  if (gridDim.y == 1) {
    for (int i = threadIdx.x; i < S * 64; i += kThreads)
      write_four(o, (i >> 6) / CT, (i >> 6) % CT, i & 63, sum_waves<WK, S>(part, i >> 6, i & 63));
    return;
  }
  // [row group][part][S][64]
  const __amdgpu_buffer_rsrc_t all_parts = __builtin_amdgcn_make_buffer_rsrc(
      parts + (int64_t)blockIdx.x * gridDim.y * S * 256, 0, gridDim.y * S * 1024, 0x00020000);
  for (int i = threadIdx.x; i < S * 64; i += kThreads)
    put4(all_parts, (blockIdx.y * S * 64 + i) * 16, sum_waves<WK, S>(part, i >> 6, i & 63));
  __shared__ int arrived;
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  if (threadIdx.x == 0) {
    const int before = __hip_atomic_fetch_add(&count[blockIdx.x], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (before == (int)gridDim.y - 1)
      __hip_atomic_store(&count[blockIdx.x], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    arrived = before;
  }
  __syncthreads();
  if (arrived != (int)gridDim.y - 1) return;
  asm volatile("" ::: "memory");
  for (int i = threadIdx.x; i < S * 64; i += kThreads) {
    float4v y = get4(all_parts, i * 16);
    for (int k = 1; k < (int)gridDim.y; ++k) y += get4(all_parts, (k * S * 64 + i) * 16);
    write_four(o, (i >> 6) / CT, (i >> 6) % CT, i & 63, y);
  }
}

template <int G, int RT, int W>
void start_gemv(const Q4Dev& m, const uint16_t* X, int64_t ldx, int B, void* Y, bool out_f32, hipStream_t s) {
  const int NT = (m.n_out + 15) / 16;
  q4_gemv_kernel<G, RT, W><<<(NT + RT - 1) / RT, 64 * W, 0, s>>>(
      m.codes, reinterpret_cast<const uint32_t*>(m.params), X, ldx, m.n_out, m.n_in, B, Y, out_f32 ? 1 : 0);
}

// Row groups that K is ever split for, and into how many parts.
constexpr int kMaxGroups = 256, kMaxParts = 8;
// The parts begin behind every count that any operator keeps, so that one
// workspace serves products and attention.
constexpr size_t kCountBytes = TQ_WORKSPACE_COUNT_BYTES;
static_assert(4 * kMaxGroups <= kCountBytes, "all counts at the front");

template <int G, int CT, int WK, int WR, int RT>
hipError_t start_gemm(const Q4Dev& m, const uint16_t* X, int64_t ldx, int B, void* Y, bool out_f32, int split, void* ws,
                      hipStream_t s) {
  const int NT = (m.n_out + 15) / 16, groups = (NT + WR * RT - 1) / (WR * RT);
  constexpr int kStage = 2 * 16 * CT * (128 * WK + 8) * 2, kPart = WK * WR * RT * CT * 64 * 16;
  constexpr int kLds = kStage > kPart ? kStage : kPart;
  static_assert(kLds <= 160 * 1024 - 64, "the LDS of a CU");
  const auto kernel = &q4_gemm_kernel<G, CT, WK, WR, RT>;
  static std::atomic<bool> set[64];   // per device: the kernel's limit of LDS is raised
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= 64 || !set[dev].load(std::memory_order_relaxed)) {
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    if (e != hipSuccess) return e;
    if (dev >= 0 && dev < 64) set[dev].store(true, std::memory_order_relaxed);
  }
  kernel<<<dim3(groups, split), 64 * WK * WR, kLds, s>>>(
      m.codes, reinterpret_cast<const uint32_t*>(m.params), X, ldx, m.n_out, m.n_in, B, Y, out_f32 ? 1 : 0,
      static_cast<int32_t*>(ws), ws ? reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + kCountBytes) : nullptr);
  return hipSuccess;
}

// What a call of B > 16 rows uses: the row tiles of a workgroup, which share its
// X, and the parts K is split into, so that few row groups fill the chip.
//   B = 64, us: 4096 x 12288 39.4 in one part, 25.2 in four (44.7 in eight); 65536
//   x 4096 101 with four row tiles, 71 with eight (one wave two of them; groups
//   of 32 have no registers for that); 12288 x 4096 25.9 and 31
struct Shape {
  int tiles, split;
};
Shape shape_of(const Q4Dev& m, int B) {
  const int NT = (m.n_out + 15) / 16, KB = (m.n_in + 127) / 128;
  Shape h = {B > 32 && NT >= 2048 && m.group > 32 ? 8 : 4, 1};
  const int groups = (NT + h.tiles - 1) / h.tiles;
  if (groups <= kMaxGroups) {
    h.split = 256 / groups;
    if (h.split > KB / 8) h.split = KB / 8;
    if (h.split > kMaxParts) h.split = kMaxParts;
    if (h.split < 1) h.split = 1;
  }
  return h;
}

template <int G>
hipError_t start_g(const Q4Dev& m, const uint16_t* X, int64_t ldx, int B, void* Y, bool out_f32, void* ws,
                   hipStream_t s) {
  const int NT = (m.n_out + 15) / 16;
  // Up to 512 row tiles (two a CU) the waves of a workgroup divide K among
  // them; beyond that they also take several row tiles, which share X.
  //   B = 1, waves x row tiles, us: 4096 x 12288 8x1 8.8, 4x2 15; 12288 x 4096 8x1
  //   11, 4x2 8.6, 4x4 10.4; 28000 x 4096 8x1 16, 4x2 13.3, 4x4 13.7; 131072 x 4096
  //   4x2 65, 4x4 54, 8x4 65
  //   B = 16, waves along K x row tiles: 4096 x 12288 16x1 11.2, 8x1 14, 4x4 21;
  //   12288 x 4096 16x1 15, 4x4 10.2; 131072 x 4096 8x1 105, 8x2 96, 4x4 76
  const bool wide = NT > 512;
  if (B <= 2 || (B <= 4 && !wide)) {
    if (NT >= 2048)
      start_gemv<G, 4, 4>(m, X, ldx, B, Y, out_f32, s);
    else if (wide)
      start_gemv<G, 2, 4>(m, X, ldx, B, Y, out_f32, s);
    else
      start_gemv<G, 1, 8>(m, X, ldx, B, Y, out_f32, s);
    return hipSuccess;
  }
  if (B <= 16)
    return wide ? start_gemm<G, 1, 4, 4, 1>(m, X, ldx, B, Y, out_f32, 1, nullptr, s)
                : start_gemm<G, 1, 16, 1, 1>(m, X, ldx, B, Y, out_f32, 1, nullptr, s);
  const Shape h = shape_of(m, B);
  const int split = ws != nullptr ? h.split : 1;
  if (B <= 32) return start_gemm<G, 2, 4, 2, 2>(m, X, ldx, B, Y, out_f32, split, ws, s);
  if constexpr (G > 32)
    if (h.tiles == 8) return start_gemm<G, 4, 2, 4, 2>(m, X, ldx, B, Y, out_f32, split, ws, s);
  return start_gemm<G, 4, 2, 4, 1>(m, X, ldx, B, Y, out_f32, split, ws, s);
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

size_t q4_workspace_bytes(const Q4Dev& m, int B) {
  if (B <= 16) return 0;
  const Shape h = shape_of(m, B);
  const size_t NT = (m.n_out + 15) / 16, groups = (NT + h.tiles - 1) / h.tiles;
  return h.split > 1 ? kCountBytes + groups * h.split * h.tiles * (B <= 32 ? 2 : 4) * 1024 : 0;
}

hipError_t launch_q4_gemm(const Q4Dev& m, const uint16_t* X, int64_t ldx, int B, void* Y, bool out_f32, void* ws,
                          hipStream_t s) {
  const hipError_t e = m.group == 32   ? start_g<32>(m, X, ldx, B, Y, out_f32, ws, s)
                       : m.group == 64 ? start_g<64>(m, X, ldx, B, Y, out_f32, ws, s)
                                       : start_g<128>(m, X, ldx, B, Y, out_f32, ws, s);
  return e != hipSuccess ? e : hipGetLastError();
}

}  // namespace tq
