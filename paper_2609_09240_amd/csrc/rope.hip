// Rotary positions (gfx950): channel pairs of a head turned by an angle of the
// token's position on the pair's axis,
//     (x1, x2) -> scale (x1 cos a - x2 sin a, x2 cos a + x1 sin a).
//
// Bound by memory where there are many tokens: every channel is read and written once
// (8191 tokens of 32 + 8 heads of 128, 168 MB: 35 us on three axes, 4.8 TB/s, 32 on
// one).  Few tokens are bound by trips to memory one behind the other: of each of a
// thread's eight pairs the axis, if it is given, and the position there, before any
// channel is loaded (1 token 5.4 us, 5.8 on three axes; 64 tokens 5.5 and 5.9).  A thread takes V pairs of one token for
// several heads, so that its V angles are formed once for them: formed for every
// two heads they take 55 us.  Four heads are loaded at a time, 8 or 10 are no
// faster.  An angle is a product in 64 bits, reduced to a fraction of a turn there
// (what a position of 10^6 leaves of a product in 32 bits is 0.06), then sine and
// cosine in 32 bits.
//
// Stores past the caches take 33 instead of 43 us where inputs come from HBM, but
// what reads the outputs next then takes longer by more than that: 72 instead of
// 68 us for both, at 1024 tokens 15.0 instead of 14.3.

#include "decode_internal.h"

namespace tq {
namespace {

struct RopeArgs {
  const int32_t* pos;
  const float* freq;
  const uint8_t* axis;
  const uint16_t *q, *k;
  uint16_t *qo, *ko;
  int64_t axis_stride, q_ts, q_hs, k_ts, k_hs, qo_ts, qo_hs, ko_ts, ko_hs;
  int32_t n_tokens, n_heads, heads, half, rot, n_axes;
  int32_t turning, units;   // threads of a token that turn V pairs each, and with those that copy V channels
  int32_t tokens, per;      // of a workgroup, and heads
  float scale, sign;
};

template <int V>
struct __attribute__((packed, aligned(2))) Some {
  _Float16 v[V];
};

template <int V, int HEADS, bool ADJACENT>
__global__ void __launch_bounds__(256) rope_kernel(RopeArgs a) {
  const int tl = threadIdx.x / a.units, u = threadIdx.x - tl * a.units + 256 * blockIdx.z;
  const int64_t t = (int64_t)blockIdx.x * a.tokens + tl;
  if (tl >= a.tokens || u >= a.units || t >= a.n_tokens) return;
  const int from_head = blockIdx.y * a.per, to_head = min(from_head + a.per, a.heads);
  auto from = [&](int h) { return h < a.n_heads ? a.q + t * a.q_ts + h * a.q_hs : a.k + t * a.k_ts + (h - a.n_heads) * a.k_hs; };
  auto to = [&](int h) { return h < a.n_heads ? a.qo + t * a.qo_ts + h * a.qo_hs : a.ko + t * a.ko_ts + (h - a.n_heads) * a.ko_hs; };
  if (u >= a.turning) {
    const int d = a.rot + (u - a.turning) * V;
    for (int h = from_head; h < to_head; ++h)
      *reinterpret_cast<Some<V>*>(to(h) + d) = *reinterpret_cast<const Some<V>*>(from(h) + d);
    return;
  }
  const int i0 = u * V;
  const int d1 = ADJACENT ? 2 * i0 : i0, d2 = ADJACENT ? 2 * i0 + V : i0 + a.half;
  float c[V], s[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int ax = a.axis ? a.axis[i0 + i] : 0;
    const int p = ax < a.n_axes ? a.pos[ax * a.axis_stride + t] : 0;
    const double turns = (double)p * (double)a.freq[i0 + i] * 0.15915494309189533577;
    sincospif(2.0f * (float)(turns - rint(turns)), &s[i], &c[i]);
    s[i] *= a.scale * a.sign;
    c[i] *= a.scale;
  }
  for (int h0 = from_head; h0 < to_head; h0 += HEADS) {
    Some<V> x[HEADS][2];
#pragma unroll
    for (int e = 0; e < HEADS; ++e) {
      const uint16_t* p = from(min(h0 + e, to_head - 1));
      x[e][0] = *reinterpret_cast<const Some<V>*>(p + d1);
      x[e][1] = *reinterpret_cast<const Some<V>*>(p + d2);
    }
#pragma unroll
    for (int e = 0; e < HEADS; ++e) {
      if (h0 + e >= to_head) break;
      Some<V> y[2];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        // Pair i: element i of either, or elements 2i and 2i + 1 of both as one.
        const float x1 = ADJACENT ? (float)x[e][2 * i / V].v[2 * i % V] : (float)x[e][0].v[i];
        const float x2 = ADJACENT ? (float)x[e][(2 * i + 1) / V].v[(2 * i + 1) % V] : (float)x[e][1].v[i];
        const _Float16 y1 = (_Float16)fmaf(x1, c[i], -(x2 * s[i])), y2 = (_Float16)fmaf(x2, c[i], x1 * s[i]);
        if (ADJACENT) {
          y[2 * i / V].v[2 * i % V] = y1;
          y[(2 * i + 1) / V].v[(2 * i + 1) % V] = y2;
        } else {
          y[0].v[i] = y1;
          y[1].v[i] = y2;
        }
      }
      uint16_t* p = to(h0 + e);
      *reinterpret_cast<Some<V>*>(p + d1) = y[0];
      *reinterpret_cast<Some<V>*>(p + d2) = y[1];
    }
  }
}

template <int V, int HEADS>
hipError_t start(const RopeArgs& a, bool adjacent, hipStream_t s) {
  const dim3 grid((a.n_tokens + a.tokens - 1) / a.tokens, (a.heads + a.per - 1) / a.per, (a.units + 255) / 256);
  if (adjacent)
    rope_kernel<V, HEADS, true><<<grid, 256, 0, s>>>(a);
  else
    rope_kernel<V, HEADS, false><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const tq_rope_call& c, hipStream_t s) {
  RopeArgs a;
  a.pos = c.positions;
  a.freq = c.freq;
  a.axis = c.axis;
  a.q = c.q.data;
  a.k = c.k.data;
  a.qo = c.q_out.data;
  a.ko = c.k_out.data;
  a.axis_stride = c.axis_stride;
  a.q_ts = c.q.token_stride, a.q_hs = c.q.head_stride;
  a.k_ts = c.k.token_stride, a.k_hs = c.k.head_stride;
  a.qo_ts = c.q_out.token_stride, a.qo_hs = c.q_out.head_stride;
  a.ko_ts = c.k_out.token_stride, a.ko_hs = c.k_out.head_stride;
  a.n_tokens = c.n_tokens;
  a.n_heads = c.n_heads;
  a.heads = c.n_heads + c.n_kv_heads;
  a.half = c.rot / 2;
  a.rot = c.rot;
  a.n_axes = c.n_axes;
  a.scale = c.scale;
  a.sign = c.flags & TQ_ROPE_INVERSE ? -1.0f : 1.0f;
  const bool in_place = c.q.data == c.q_out.data && (c.n_kv_heads == 0 || c.k.data == c.k_out.data);
  const int rest = in_place ? 0 : c.head_dim - c.rot;
  auto fits = [&](int v) { return a.half % v == 0 && rest % v == 0; };
  const int V = fits(8) ? 8 : fits(4) ? 4 : fits(2) ? 2 : 1;
  a.turning = a.half / V;
  a.units = a.turning + rest / V;
  a.tokens = a.units <= 256 ? 256 / a.units : 1;
  // Heads of a workgroup: four where there are few tokens, eight where fours would
  // make more than 2.5 workgroups a CU (32 + 8 heads of 128 from HBM, with 4, 8, 20
  // heads: 256 tokens 5.7, 7.2, 11.5 us; 2048: 14.7, 14.6, 19.2; 8191: 43.7, 40.4,
  // 44.1, from caches 41, 35, 35; all of them on one axis, without an array of axes).
  const int64_t fours = (int64_t)((a.n_tokens + a.tokens - 1) / a.tokens) * ((a.heads + 3) / 4);
  a.per = fours < 640 ? 4 : 8;
  const bool adjacent = c.flags & TQ_ROPE_ADJACENT;
  if (V == 8) return start<8, 4>(a, adjacent, s);
  if (V == 4) return start<4, 4>(a, adjacent, s);
  if (V == 2) return start<2, 4>(a, adjacent, s);
  return start<1, 4>(a, adjacent, s);
}

}  // namespace tq
