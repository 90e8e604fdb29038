// Log probabilities of rows of logits (gfx950), one pass over them:
//     m = max x, S = sum exp(scale (x - m)), T = sum exp(scale (x - m)) (x - m),
//     log p_j = scale (x_j - m) - log S,   H = log S - scale T / S,
// with the sums rescaled whenever a thread's maximum grows (x - m <= 0, so
// neither term of H cancels the other).
//
// The most likely tokens.  A wave holds a chunk of 1024 logits in registers.  The
// k-th largest of its 64 lanes' maxima bounds the k-th largest logit from below,
// so that few others have to be looked at: those above the bound, and of those
// equal to it the first k.  They go to LDS as whole numbers (order of the logit,
// then of the index) and are ranked by counting.  In later chunks only what is
// above the k-th so far is looked at, mostly nothing.
//
// A workgroup takes a row or, where there are few rows, a part of one; the last
// workgroup of a row to leave its part joins them in their order.

#include "decode_internal.h"

namespace tq {
namespace {

constexpr int kEach = 16, kThreads = 256, kChunk = kThreads * kEach;
constexpr int kMaxParts = 16, kMaxTop = TQ_LOGPROBS_MAX_TOP;
constexpr int kPartFloats = 4 + 2 * kMaxTop;   // m, S, T, unused, keys
constexpr int kWanted = 2048;                  // workgroups
// Candidates of a wave: what it held, those above the bound in fewer than k
// lanes, the first k equal to it.
constexpr int kMost = kMaxTop + (kMaxTop - 1) * kEach + kMaxTop;
constexpr float kLowest = -3.4028234663852886e38f;   // of the finite numbers

struct LogArgs {
  const void* x;
  int64_t ld;
  const int32_t* ids;
  float *logp, *entropy, *top_logp;
  int32_t *top_ids, *d_err, *count;
  float* part;
  int32_t V, n_ids, k, parts, chunks, rows;   // chunks of a part
  float scale;
};

// The order of logits as that of whole numbers, the index below: larger logits
// first, of equal ones the lower index.
__device__ inline uint64_t key_of(float x, int j) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);
  const uint32_t o = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
  return ((uint64_t)o << 32) | (uint32_t)~j;
}
__device__ inline float logit_of(uint64_t key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __builtin_bit_cast(float, o ^ (o & 0x80000000u ? 0x80000000u : 0xFFFFFFFFu));
}

struct Sums {
  float m, s, t;
};
__device__ inline Sums join(Sums a, Sums b, float c) {
  Sums r;
  r.m = fmaxf(a.m, b.m);
  const float m = fmaxf(r.m, kLowest);
  const float da = fmaxf(fmaxf(a.m, kLowest) - m, kLowest), db = fmaxf(fmaxf(b.m, kLowest) - m, kLowest);
  const float fa = __builtin_amdgcn_exp2f(da * c), fb = __builtin_amdgcn_exp2f(db * c);
  const float sa = a.s * fa, sb = b.s * fb;
  r.s = sa + sb;
  r.t = fmaf(sa, da, a.t * fa) + fmaf(sb, db, b.t * fb);
  return r;
}

__device__ inline int below(uint64_t mask) {   // lanes of a mask before this one
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// What a wave wrote to LDS is there for all its lanes.
__device__ inline void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The k-th largest of the 64 lanes' x (none of them NaN).
__device__ inline float kth_of(float x, int k) {
  int rank = 0;
  const int lane = threadIdx.x & 63;
#pragma unroll 8
  for (int i = 0; i < 64; ++i) {
    const float y = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), i));
    rank += y > x || (y == x && i < lane);
  }
  const int at = __ffsll((unsigned long long)__builtin_amdgcn_ballot_w64(rank == k - 1)) - 1;
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), at));
}

// The largest keys of a wave's part of a row, in LDS: `list` (n of them, the first k in
// order between chunks), and what an unseen logit has to be above.
struct Top {
  uint64_t* list;
  uint64_t* sorted;
  int n;
  float bound;
};

__device__ inline void rank_keys(Top& top, int k) {
  const int lane = threadIdx.x & 63;
  wave_sync();
  for (int i = lane; i < top.n; i += 64) {
    const uint64_t mine = top.list[i];
    int rank = 0;
    for (int j = 0; j < top.n; ++j) rank += top.list[j] > mine;
    if (rank < k) top.sorted[rank] = mine;
  }
  wave_sync();
  if (lane < k) top.list[lane] = top.sorted[lane];
  wave_sync();
  top.n = k;
  top.bound = logit_of(top.list[k - 1]);
}

template <class T>
struct __attribute__((packed, aligned(sizeof(T)))) Vec {
  T v[16 / sizeof(T)];
};

template <class T, bool ENTROPY, bool TOP>
__global__ void __launch_bounds__(kThreads) logprobs_kernel(LogArgs a) {
  constexpr int VE = 16 / sizeof(T), NV = kEach / VE;
  __shared__ uint64_t list[TOP ? kThreads / 64 : 1][TOP ? kMost : 1];
  alignas(16) __shared__ uint64_t best[TOP ? kMaxParts * kMaxTop : 1];
  __shared__ Sums sums[kThreads / 64];
  __shared__ int last;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts;
  const T* x = static_cast<const T*>(a.x) + row * a.ld;
  const float c = a.scale * 1.4426950408889634f;
  const int k = TOP ? a.k : 0;
  Sums z = {-__builtin_inff(), 0.0f, 0.0f};
  Top top = {list[TOP ? wave : 0], best + (TOP ? wave * kMaxTop : 0), 0, -__builtin_inff()};

  const int c0 = part * a.chunks;
  for (int chunk = c0; chunk < c0 + a.chunks && chunk * kChunk < a.V; ++chunk) {
    float v[kEach];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = chunk * kChunk + (i * kThreads + tid) * VE;
      if (j + VE <= a.V) {
        const Vec<T> w = *reinterpret_cast<const Vec<T>*>(x + j);
#pragma unroll
        for (int e = 0; e < VE; ++e) v[i * VE + e] = (float)w.v[e];
      } else {
#pragma unroll
        for (int e = 0; e < VE; ++e) v[i * VE + e] = j + e < a.V ? (float)x[j + e] : -__builtin_inff();
      }
    }
    float most = -__builtin_inff();
#pragma unroll
    for (int e = 0; e < kEach; ++e) most = fmaxf(most, v[e]);
    {
      const float now = fmaxf(z.m, most), m = fmaxf(now, kLowest), by = fmaxf(fmaxf(z.m, kLowest) - m, kLowest);
      const float f = __builtin_amdgcn_exp2f(by * c);
      z.s *= f;
      if (ENTROPY) z.t = fmaf(z.s, by, z.t * f);
      z.m = now;
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const float d = v[e] - m, p = __builtin_amdgcn_exp2f(d * c);
        z.s += p;
        if (ENTROPY) z.t = fmaf(p, fmaxf(d, kLowest), z.t);   // 0 times -infinity
      }
    }
    if constexpr (TOP) {
      const bool first = chunk == c0;
      const uint64_t above = __builtin_amdgcn_ballot_w64(most > top.bound);
      if (!first && above == 0) continue;
      const bool equal = first || __popcll(above) >= k;
      if (equal) top.bound = kth_of(most, k);
      int n = top.n;
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const uint64_t mask = __builtin_amdgcn_ballot_w64(v[e] > top.bound);
        if (mask == 0) continue;
        const int j = chunk * kChunk + (e / VE * kThreads + tid) * VE + e % VE;
        if (v[e] > top.bound) top.list[n + below(mask)] = key_of(v[e], j);
        n += __popcll(mask);
      }
      int ties = 0;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (!equal || ties >= k) break;
        int mine = 0;
        // (a NaN ranks as -infinity)
#pragma unroll
        for (int e = 0; e < VE; ++e) mine += fmaxf(v[i * VE + e], -__builtin_inff()) == top.bound;
        if (__builtin_amdgcn_ballot_w64(mine != 0) == 0) continue;
        const int incl = wave_scan(mine);
        int at = ties + incl - mine;
#pragma unroll
        for (int e = 0; e < VE; ++e)
          if (fmaxf(v[i * VE + e], -__builtin_inff()) == top.bound) {
            if (at < k) top.list[n + at] = key_of(top.bound, chunk * kChunk + (i * kThreads + tid) * VE + e);
            ++at;
          }
        ties += __builtin_amdgcn_readlane(incl, 63);
      }
      top.n = n + min(ties, k);
      rank_keys(top, k);
    }
  }

  // The workgroup's sums and keys.
#pragma unroll
  for (int d = 1; d < 64; d *= 2) z = join(z, Sums{__shfl_xor(z.m, d), __shfl_xor(z.s, d), __shfl_xor(z.t, d)}, c);
  if (lane == 0) sums[wave] = z;
  __syncthreads();
  z = sums[0];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) z = join(z, sums[w], c);
  auto rank_all = [&](int n) {   // keys in list[0][0 .. n) to best[0 .. k), from largest
    for (int i = tid; i < n; i += kThreads) {
      const uint64_t mine = list[0][i];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += list[0][j] > mine;
      if (rank < k) best[rank] = mine;
    }
    __syncthreads();
  };
  if constexpr (TOP) {
    const uint64_t mine = tid < 4 * k ? list[tid / k][tid % k] : 0;
    __syncthreads();
    if (tid < 4 * k) list[0][tid] = mine;
    __syncthreads();
    rank_all(4 * k);
  }

  if (a.parts > 1) {
    const __amdgpu_buffer_rsrc_t parts_of =
        __builtin_amdgcn_make_buffer_rsrc(a.part, 0, a.rows * a.parts * kPartFloats * 4, 0x00020000);
    const int at = blockIdx.x * kPartFloats * 4;
    if (tid == 0) put4(parts_of, at, float4v{z.m, z.s, z.t, 0.0f});
    if constexpr (TOP)
      if (tid < (k + 1) / 2) {
        const u4v w = *reinterpret_cast<const u4v*>(&best[2 * tid]);
        put4(parts_of, at + 16 + 16 * tid, __builtin_bit_cast(float4v, w));
      }
    __builtin_amdgcn_s_waitcnt(0);   // what is joined has arrived
    __syncthreads();
    if (tid == 0) {
      const int before = __hip_atomic_fetch_add(a.count + row, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (before == a.parts - 1) __hip_atomic_store(a.count + row, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      last = before == a.parts - 1;
    }
    __syncthreads();
    if (!last) return;
    asm volatile("" ::: "memory");
    const int at0 = row * a.parts * kPartFloats * 4;
    for (int p = 0; p < a.parts; ++p) {
      const float4v w = get4(parts_of, at0 + p * kPartFloats * 4);
      const Sums y = {w[0], w[1], w[2]};
      z = p == 0 ? y : join(z, y, c);
    }
    if constexpr (TOP) {
      const int pairs = (k + 1) / 2;
      for (int i = tid; i < a.parts * pairs; i += kThreads) {
        const int p = i / pairs, e = i - p * pairs;
        const u4v w = __builtin_bit_cast(u4v, get4(parts_of, at0 + p * kPartFloats * 4 + 16 + 16 * e));
        list[0][p * k + 2 * e] = (uint64_t)w[1] << 32 | w[0];
        if (2 * e + 1 < k) list[0][p * k + 2 * e + 1] = (uint64_t)w[3] << 32 | w[2];
      }
      __syncthreads();
      rank_all(a.parts * k);
    }
  }

  // What is asked for.  Where no token is possible S is 0.
  const bool none = z.s == 0.0f;
  const float log_s = logf(z.s);
  auto logp = [&](float v) { return none ? -__builtin_inff() : (v - z.m) * a.scale - log_s; };
  for (int i = tid; i < a.n_ids; i += kThreads) {
    const int64_t at = (int64_t)row * a.n_ids + i;
    const int id = a.ids[at];
    const bool in = id >= 0 && id < a.V;
    a.logp[at] = in ? logp((float)x[id]) : __builtin_nanf("");
    if (!in && a.d_err != nullptr) atomicAdd(a.d_err, 1);
  }
  if (ENTROPY && tid == 0) a.entropy[row] = none ? 0.0f : log_s - a.scale * z.t / z.s;
  if constexpr (TOP) {
    if (tid < k) {
      const uint64_t key = best[tid];
      a.top_ids[(int64_t)row * k + tid] = (int)~(uint32_t)key;
      a.top_logp[(int64_t)row * k + tid] = logp(logit_of(key));
    }
  }
}

// Parts of a row, and chunks of one: as many workgroups as fill the chip, whole
// chunks each.
void split(const tq_logprobs_call& c, int* parts, int* chunks) {
  const int all = (c.n_vocab + kChunk - 1) / kChunk;
  int p = (kWanted + c.n_rows - 1) / c.n_rows;
  p = p < all ? p : all;
  p = p < kMaxParts ? p : kMaxParts;
  *chunks = (all + p - 1) / p;
  *parts = (all + *chunks - 1) / *chunks;
}
static_assert(kWanted * 4 <= TQ_WORKSPACE_COUNT_BYTES, "rows that are split have a count each");

template <class T>
void start(const LogArgs& a, hipStream_t s) {
  const dim3 grid(a.rows * a.parts);
  if (a.k > 0) {
    if (a.entropy != nullptr)
      logprobs_kernel<T, true, true><<<grid, kThreads, 0, s>>>(a);
    else
      logprobs_kernel<T, false, true><<<grid, kThreads, 0, s>>>(a);
  } else {
    if (a.entropy != nullptr)
      logprobs_kernel<T, true, false><<<grid, kThreads, 0, s>>>(a);
    else
      logprobs_kernel<T, false, false><<<grid, kThreads, 0, s>>>(a);
  }
}

}  // namespace

size_t logprobs_workspace_bytes(const tq_logprobs_call& c) {
  int parts, chunks;
  split(c, &parts, &chunks);
  return parts > 1 ? TQ_WORKSPACE_COUNT_BYTES + (size_t)c.n_rows * parts * kPartFloats * 4 : 0;
}

hipError_t launch_logprobs(const tq_logprobs_call& c, hipStream_t s) {
  LogArgs a;
  split(c, &a.parts, &a.chunks);
  a.x = c.logits;
  a.ld = c.ld;
  a.ids = c.ids;
  a.logp = c.logp;
  a.entropy = c.entropy;
  a.top_logp = c.top_logp;
  a.top_ids = c.top_ids;
  a.d_err = c.d_err;
  a.count = static_cast<int32_t*>(c.workspace);
  a.part = c.workspace != nullptr
               ? reinterpret_cast<float*>(static_cast<uint8_t*>(c.workspace) + TQ_WORKSPACE_COUNT_BYTES)
               : nullptr;
  a.V = c.n_vocab;
  a.n_ids = c.n_ids;
  a.k = c.n_top;
  a.rows = c.n_rows;
  a.scale = c.scale;
  if (c.flags == TQ_LOGITS_FP32)
    start<float>(a, s);
  else
    start<_Float16>(a, s);
  return hipGetLastError();
}

}  // namespace tq
