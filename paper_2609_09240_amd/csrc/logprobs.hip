// Log probabilities of rows of logits (gfx950), one pass over them.  With t_j =
// scale log2(e) (x_j - m), where m is the largest of them,
//     S = sum 2^t_j,  T = sum 2^t_j t_j,
//     log p_j = scale (x_j - m) - log S,   H = log S - ln 2 T / S;
// m moves, and the sums with it, whenever a wave's maximum grows.
//
// The most likely tokens.  A wave holds 1024 logits in registers.  The k-th
// largest of its 64 lanes' maxima bounds the k-th largest logit from below, and
// so does the largest such bound of the workgroup's waves: few logits reach it.
// Those above it, and of those equal to it the first k of the wave, go to LDS as
// whole numbers (order of the logit, then of the index), and are ranked by
// counting, once for a workgroup.  In later chunks only what is above the bound is
// looked at.
//
// A workgroup takes a row or, where there are few rows, a part of one; the last
// workgroup of a row to leave its part joins them in their order.
//
// Bound by memory where rows are many and long: 1500 rows of 49999 fp16 logits
// (150 MB) with the most likely one 46 us, 3.2 TB/s, of which vector instructions
// are about 29; without 38.  Few rows: 64 of 131072 fp32 logits (34 MB) 21 us with the
// 20 most likely ones, 13.4 without: a part has two chunks, between which the whole
// workgroup ranks; one row of 131072 fp16 logits in 16 parts 14.  1 row of 5000 6.8:
// launch, two chunks in one workgroup, ranking after either.

#include "decode_internal.h"

namespace tq {
namespace {

constexpr int kEach = 16, kThreads = 256, kWaves = kThreads / 64, kChunk = kThreads * kEach;
constexpr int kMaxParts = 16, kMaxTop = TQ_LOGPROBS_MAX_TOP;
constexpr int kPartFloats = 4 + 2 * kMaxTop;   // reference and its logit, S, T, keys
constexpr int kWanted = 2048;                  // workgroups
// Candidates of a wave: what it held when a chunk began (ranked, and k left of
// them, where it was more than kHeld), those above the bound in fewer than k
// lanes, the first k equal to it.
constexpr int kHeld = 64, kMost = kHeld + (kMaxTop - 1) * kEach + kMaxTop;
static_assert(kMaxParts * kMaxTop <= kMost && kMost % 8 == 0, "the join's keys, and ranking by eights");
constexpr float kLowest = -3.4028234663852886e38f;   // of the finite numbers
constexpr float kLn2 = 0.69314718055994531f;

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

// Half of x - m, which is finite where both are: 3e38 and -3e38 are 6e38 apart.
__device__ inline float half_of(float x, float m) { return fmaf(0.5f, x, -0.5f * m); }

// A logit relative to a reference, in powers of two; c2 is twice scale log2(e).
// (x - m) c and not x c - m c: where scales are large or logits far from 0 what
// m c loses when it is rounded would be more than there is between them.  (For 1500
// rows of 49999 fp16 logits, where x - m is almost always exact, it cost 1 to 2.7 us
// of 46.)
struct Ref {
  float c2, m;
  __device__ Ref(float m, float c2) : c2(c2), m(fmaxf(m, kLowest)) {}
  __device__ float operator()(float x) const { return half_of(x, m) * c2; }
  __device__ float from(const Ref& o) const { return half_of(o.m, m) * c2; }   // of o's reference
};

// Largest logit m, S - 1 and T against it: one of the logits that equal m is left
// out of the sum, whose term is 1: the log probability of a token that is nearly
// certain is that of the others' sum, which the steps of a sum near 1 would drown,
// wherever those others lie.
struct Sums {
  float m, s, t;
  __device__ float all() const { return (m > -__builtin_inff() ? 1.0f : 0.0f) + s; }
};
__device__ inline Sums join(Sums a, Sums b, float c2) {
  const bool first = a.m >= b.m;
  const Sums w = first ? a : b, l = first ? b : a;
  const float by = fmaxf(Ref(w.m, c2).from(Ref(l.m, c2)), kLowest), f = __builtin_amdgcn_exp2f(by), s = l.all() * f;
  return Sums{w.m, w.s + s, w.t + fmaf(s, by, l.t * f)};
}

__device__ inline int below(uint64_t mask) {   // lanes of a mask before this one
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// What a wave wrote to LDS is there for all its lanes.
__device__ inline void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

__device__ inline float lane_of(float x, int i) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), i));
}

// One step of a sort of the lanes: of lanes whose numbers differ in bit J, the
// one whose bit J is not that of the direction (bit K) takes the larger x.
template <int J, int K>
__device__ inline void sort_step(float& x, int lane) {
  const int b = __builtin_bit_cast(int, x);
  float y = x, z;
  if constexpr (J >= 16) {   // both of a pair, in either lane
    const auto w = J == 16 ? __builtin_amdgcn_permlane16_swap(b, b, false, false)
                           : __builtin_amdgcn_permlane32_swap(b, b, false, false);
    const uint32_t w0 = w[0], w1 = w[1];   // (a bit cast of a vector's element takes its first one)
    y = __builtin_bit_cast(float, w0);
    z = __builtin_bit_cast(float, w1);
  } else if constexpr (J == 4) {   // lanes 4 up in the quads 0 and 2 of a row, 4 down in 1 and 3
    const int w = __builtin_amdgcn_update_dpp(0, b, 0x104, 0xF, 0x5, false);
    z = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(w, b, 0x114, 0xF, 0xA, false));
  } else {   // quad_perm 1 0 3 2 and 2 3 0 1, row_ror 8
    z = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, b, J == 1 ? 0xB1 : J == 2 ? 0x4E : 0x128, 0xF, 0xF, true));
  }
  const bool smaller = ((lane & J) != 0) != ((lane & K) != 0);
  x = smaller ? fminf(y, z) : fmaxf(y, z);
}
template <int J, int K>
__device__ inline void sort_steps(float& x, int lane) {
  sort_step<J, K>(x, lane);
  if constexpr (J > 1) sort_steps<J / 2, K>(x, lane);
}

// The k-th largest of the 64 lanes' x (none of them NaN): they are sorted, the
// largest in lane 0.
__device__ inline float kth_of(float x, int k) {
  const int lane = threadIdx.x & 63;
  sort_steps<1, 2>(x, lane);
  sort_steps<2, 4>(x, lane);
  sort_steps<4, 8>(x, lane);
  sort_steps<8, 16>(x, lane);
  sort_steps<16, 32>(x, lane);
  sort_steps<32, 64>(x, lane);
  return lane_of(x, k - 1);
}

// The largest of the lanes' x, uniform.
template <int CTRL>
__device__ inline float max_dpp(float x) {
  const int b = __builtin_bit_cast(int, x);
  return fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(b, b, CTRL, 0xF, 0xF, true)));
}
__device__ inline float wave_max(float x) {
  x = max_dpp<0xB1>(x);    // quad_perm 1 0 3 2
  x = max_dpp<0x4E>(x);    // quad_perm 2 3 0 1
  x = max_dpp<0x141>(x);   // row_half_mirror
  x = max_dpp<0x140>(x);   // row_mirror
  uint32_t b = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
  uint32_t r0 = r[0], r1 = r[1];
  b = __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, r0), __builtin_bit_cast(float, r1)));
  const auto w = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  r0 = w[0], r1 = w[1];
  return lane_of(fmaxf(__builtin_bit_cast(float, r0), __builtin_bit_cast(float, r1)), 0);
}

// Keys of a list of n, filled up with zeros to a multiple of 8, above one.
__device__ inline int rank_in(const uint64_t* list, int n, uint64_t mine) {
  int rank = 0;
  for (int j = 0; j < n; j += 8) {
    u4v w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = *reinterpret_cast<const u4v*>(&list[j + 2 * e]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      rank += ((uint64_t)w[e][1] << 32 | w[e][0]) > mine;
      rank += ((uint64_t)w[e][3] << 32 | w[e][2]) > mine;
    }
  }
  return rank;
}

// The first k of a wave's n keys to the front of its list, in order; the rest
// is gone.
__device__ inline void rank_wave(uint64_t* list, uint64_t* sorted, int n, int k) {
  const int lane = threadIdx.x & 63;
  if (lane < 8 && n + lane < ((n + 7) & ~7)) list[n + lane] = 0;
  wave_sync();
  for (int i = lane; i < n; i += 64) {
    const uint64_t mine = list[i];
    const int rank = rank_in(list, n, mine);
    if (rank < k) sorted[rank] = mine;
  }
  wave_sync();
  if (lane < k) list[lane] = sorted[lane];
  wave_sync();
}

template <class T>
struct __attribute__((packed, aligned(sizeof(T)))) Vec {
  T v[16 / sizeof(T)];
};

// Six waves a SIMD, 80 vector registers: fp16 with the entropy and the most likely
// tokens spills three of them, and 30 to 42 scalar ones go to lanes of vector registers.
// With five waves nothing is spilled and 1500 rows of 49999 take 60 us instead of 47.
template <class T, bool ENTROPY, bool TOP>
__global__ void __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(6))) logprobs_kernel(LogArgs a) {
  constexpr int VE = 16 / sizeof(T), NV = kEach / VE;
  alignas(16) __shared__ uint64_t list[TOP ? kWaves : 1][TOP ? kMost : 2];
  __shared__ uint64_t best[TOP ? kMaxTop + 1 : 1], sorted[TOP ? kWaves : 1][TOP ? kMaxTop : 1];
  __shared__ Sums sums[kWaves];
  __shared__ float bounds[kWaves];
  __shared__ int counts[kWaves + 1];
  __shared__ int last;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts;
  const T* x = static_cast<const T*>(a.x) + row * a.ld;
  const float c2 = lane_of(a.scale * 2.8853900817779268f, 0);   // (uniform: no vector register)
  const int k = TOP ? a.k : 0;
  const float none = -__builtin_inff();
  // The lane's sums against the largest logit of its wave, which is left out of
  // those of lane `holder`.
  Sums z = {none, 0.0f, 0.0f};
  int holder = -1;
  uint64_t* mine = list[TOP ? wave : 0];
  int held = 0;
  float bound = none;

  // Thread's logits of a chunk; past the row -infinity.
  auto load = [&](Vec<T>(&w)[NV], int chunk) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = chunk * kChunk + (i * kThreads + tid) * VE;
      if (j + VE <= a.V) {
        w[i] = *reinterpret_cast<const Vec<T>*>(x + j);
      } else {
#pragma unroll
        for (int e = 0; e < VE; ++e) w[i].v[e] = j + e < a.V ? x[j + e] : (T)none;
      }
    }
  };
  // The first k of n keys in list[0] to best, in order.
  auto rank_all = [&](int n) {
    if (tid < 8 && n + tid < ((n + 7) & ~7)) list[0][n + tid] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) {
      const uint64_t key = list[0][i];
      const int rank = rank_in(list[0], n, key);
      if (rank < k) best[rank] = key;
    }
    __syncthreads();
  };
  // The first k of all waves' keys to best, in order.
  auto rank_lists = [&] {
    if (held > kMost / kWaves) {   // all four lists fit one
      rank_wave(mine, sorted[wave], held, k);
      held = k;
    }
    if (lane == 0) counts[wave] = held;
    __syncthreads();
    int n = 0, at = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) at += counts[w];
      n += counts[w];
    }
    constexpr int kOwn = (kMost / kWaves + 63) / 64;
    uint64_t key[kOwn];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) key[i] = i * 64 + lane < held ? mine[i * 64 + lane] : 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kOwn; ++i)
      if (i * 64 + lane < held) list[0][at + i * 64 + lane] = key[i];
    __syncthreads();
    rank_all(n);
  };
  const int c0 = part * a.chunks, c1 = min(c0 + a.chunks, (a.V + kChunk - 1) / kChunk);
  Vec<T> next[NV];
  load(next, c0);
  for (int chunk = c0; chunk < c1; ++chunk) {
    float v[kEach], most = none;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      v[e] = (float)next[e / VE].v[e % VE];
      asm("" : "+v"(v[e]));   // now, so that the next chunk's loads need no registers of their own
      most = fmaxf(most, v[e]);
    }
    if (chunk + 1 < c1) load(next, chunk + 1);
    // A sum of 16 terms, of which `leaves_out` says which is none of it.
    auto add = [&](auto leaves_out) {
      const Ref r(z.m, c2);
      float sum = 0.0f;
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const float t = r(v[e]), p = __builtin_amdgcn_exp2f(t);
        sum += leaves_out(v[e]) ? 0.0f : p;
        if (ENTROPY) z.t = fmaf(p, fmaxf(t, kLowest), z.t);   // 0 times -infinity
      }
      z.s += sum;
    };
    if (__builtin_amdgcn_ballot_w64(most > z.m) == 0) {
      add([](float) { return false; });
    } else {
      const float now = wave_max(most), by = fmaxf(Ref(now, c2).from(Ref(z.m, c2)), kLowest), f = __builtin_amdgcn_exp2f(by);
      z.s = (lane == holder ? z.s + 1.0f : z.s) * f;
      if (ENTROPY) z.t = fmaf(z.s, by, z.t * f);
      z.m = now;
      // The first logit that equals it, of the first lane that has one.  (+infinity is
      // left in: its term is NaN.)
      holder = __ffsll((unsigned long long)__builtin_amdgcn_ballot_w64(most == now)) - 1;
      bool out = lane == holder && now < __builtin_inff();
      add([&](float x) {
        const bool it = out && x == now;
        out = out && !it;
        return it;
      });
    }
    if constexpr (TOP) {
      const bool first = chunk == c0;
      bool equal = first;
      if (first) {
        const float b = k == 1 ? z.m : kth_of(most, k);
        if (lane == 0) bounds[wave] = b;
        __syncthreads();
        bound = fmaxf(fmaxf(bounds[0], bounds[1]), fmaxf(bounds[2], bounds[3]));
      } else {
        const uint64_t above = __builtin_amdgcn_ballot_w64(most > bound);
        if (above == 0) continue;
        if (held > kHeld) {
          rank_wave(mine, sorted[wave], held, k);
          held = k;
          bound = fmaxf(bound, logit_of(mine[k - 1]));
        }
        if (__popcll(above) >= k) {
          const float b = kth_of(most, k);
          equal = b > bound;
          bound = fmaxf(bound, b);
        }
      }
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const uint64_t mask = __builtin_amdgcn_ballot_w64(v[e] > bound);
        if (mask == 0) continue;
        const int j = chunk * kChunk + (e / VE * kThreads + tid) * VE + e % VE;
        if (v[e] > bound) mine[held + below(mask)] = key_of(v[e], j);
        held += __popcll(mask);
      }
      int ties = 0;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (!equal || ties >= k) break;
        int n = 0;
        // (a NaN ranks as -infinity)
#pragma unroll
        for (int e = 0; e < VE; ++e) n += fmaxf(v[i * VE + e], none) == bound;
        if (__builtin_amdgcn_ballot_w64(n != 0) == 0) continue;
        const int incl = wave_scan(n);
        int at = ties + incl - n;
#pragma unroll
        for (int e = 0; e < VE; ++e)
          if (fmaxf(v[i * VE + e], none) == bound) {
            if (at < k) mine[held + at] = key_of(bound, chunk * kChunk + (i * kThreads + tid) * VE + e);
            ++at;
          }
        ties += __builtin_amdgcn_readlane(incl, 63);
      }
      held += min(ties, k);
      if (first && c1 > c0 + 1 && k > 1) {   // the bound of the whole chunk (for one token it is there)
        rank_lists();
        held = wave == 0 ? k : 0;
        if (tid < k) list[0][tid] = best[tid];
        bound = logit_of(best[k - 1]);
        __syncthreads();
      }
    }
  }

  // The workgroup's sums and keys.
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    z.s += __shfl_xor(z.s, d);
    if (ENTROPY) z.t += __shfl_xor(z.t, d);
  }
  if (lane == 0) sums[wave] = z;
  if constexpr (TOP) rank_lists();
  __syncthreads();
  z = sums[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) z = join(z, sums[w], c2);

  if (a.parts > 1) {
    const __amdgpu_buffer_rsrc_t parts_of =
        __builtin_amdgcn_make_buffer_rsrc(a.part, 0, a.rows * a.parts * kPartFloats * 4, 0x00020000);
    const int at = blockIdx.x * kPartFloats * 4;
    if (tid == 0) put4(parts_of, at, float4v{z.m, z.s, z.t, 0.0f});
    if constexpr (TOP)
      if (tid < (k + 1) / 2) {
        const uint64_t p = best[2 * tid], q = best[2 * tid + 1];
        const u4v w = {(uint32_t)p, (uint32_t)(p >> 32), (uint32_t)q, (uint32_t)(q >> 32)};
        put4(parts_of, at + 16 + 16 * tid, __builtin_bit_cast(float4v, w));
      }
    __builtin_amdgcn_s_waitcnt(0);   // what is joined has arrived
    __syncthreads();
    if (tid == 0) {
      const int before = __hip_atomic_fetch_add(a.count + row, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (before == a.parts - 1) __hip_atomic_store(a.count + row, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      last = before == a.parts - 1;
    }
    if (tid <= kWaves) counts[tid] = 0;
    __syncthreads();
    if (!last) return;
    asm volatile("" ::: "memory");
    const int at0 = row * a.parts * kPartFloats * 4;
    // Lane p of every 16 has part p's sums.
    const float4v w = get4(parts_of, at0 + min(lane & 15, a.parts - 1) * kPartFloats * 4);
    z = (lane & 15) < a.parts ? Sums{w[0], w[1], w[2]} : Sums{none, 0.0f, 0.0f};
    if constexpr (TOP) {
      // Of every part's keys the n-th, with n parts >= k: at least k keys are not
      // below the least of them.
      const int pairs = (k + 1) / 2, nth = (k + a.parts - 1) / a.parts;
      constexpr int kOwn = kMaxParts * kMaxTop / 2 / kThreads;
      static_assert(kOwn == 1, "a pair of keys a thread");
      uint64_t key[2] = {0, 0};
      const int p = tid / pairs, e = tid - p * pairs;
      if (p < a.parts) {
        const u4v y = __builtin_bit_cast(u4v, get4(parts_of, at0 + p * kPartFloats * 4 + 16 + 16 * e));
        key[0] = (uint64_t)y[1] << 32 | y[0];
        if (2 * e + 1 < k) key[1] = (uint64_t)y[3] << 32 | y[2];
        if ((nth - 1) / 2 == e) best[p] = key[(nth - 1) & 1];
      }
      __syncthreads();
      uint64_t least = best[0];
      for (int i = 1; i < a.parts; ++i) least = best[i] < least ? best[i] : least;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint64_t mask = __builtin_amdgcn_ballot_w64(key[i] != 0 && key[i] >= least);
        int first = 0;
        if (lane == 0 && mask != 0) first = atomicAdd(&counts[kWaves], __popcll(mask));
        first = __builtin_amdgcn_readfirstlane(first);
        if (key[i] != 0 && key[i] >= least) list[0][first + below(mask)] = key[i];
      }
      __syncthreads();
      rank_all(counts[kWaves]);
    }
#pragma unroll
    for (int d = 1; d < kMaxParts; d *= 2)
      z = join(z, Sums{__shfl_xor(z.m, d), __shfl_xor(z.s, d), __shfl_xor(z.t, d)}, c2);
  }

  // What is asked for.  Where no token is possible S is 0.
  const bool empty = z.all() == 0.0f;
  const float log_s = log1pf(z.s);
  auto logp = [&](float v) { return empty ? none : 2.0f * (half_of(v, z.m) * a.scale) - log_s; };
  for (int i = tid; i < a.n_ids; i += kThreads) {
    const int64_t at = (int64_t)row * a.n_ids + i;
    const int id = a.ids[at];
    const bool in = id >= 0 && id < a.V;
    a.logp[at] = in ? logp((float)x[id]) : __builtin_nanf("");
    if (!in && a.d_err != nullptr) atomicAdd(a.d_err, 1);
  }
  if (ENTROPY && tid == 0) a.entropy[row] = empty ? 0.0f : log_s - z.t / z.all() * kLn2;
  if constexpr (TOP) {
    if (tid < k) {
      const uint64_t key = best[tid];
      a.top_ids[(int64_t)row * k + tid] = (int)~(uint32_t)key;
      a.top_logp[(int64_t)row * k + tid] = logp(logit_of(key));
    }
  }
}

// Parts of a row, and chunks of one: as many workgroups as the chip holds at
// once, two chunks each at least (the second is on its way while the first is
// looked at; joining takes 3 us).
void split(const tq_logprobs_call& c, int* parts, int* chunks) {
  const int all = (c.n_vocab + kChunk - 1) / kChunk;
  int p = kWanted / c.n_rows;
  p = p < all / 2 ? p : all / 2;
  p = p < 1 ? 1 : p < kMaxParts ? p : kMaxParts;
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
