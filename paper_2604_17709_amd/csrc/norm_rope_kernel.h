// Norms of queries and keys for each head, with the rotary embedding in the same pass, and the way of keys and values
// into the cache.
//
//   y = w x / sqrt(mean over the head of x^2 + eps)           (where there is a weight for it)
//   a = positions[axis of pair i][t] * freqs[i]               (the angle of pair i, i < rot_dim / 2)
//   y_first  <- m (y_first cos a - y_second sin a)
//   y_second <- m (y_second cos a + y_first sin a)
//
// with the pair (i, i + rot_dim / 2) of a head, or (2 i, 2 i + 1) where pairs are interleaved; the elements from
// rot_dim on are normed only, values are copied.  Everything between the load and the store is fp32, with one rounding.  Bound by HBM:
// every element is read once and written once.  A workgroup has a row, as many lanes as a head has pieces a head, so that its sum of squares is a
// few exchanges between lanes and the row's cosines and sines are formed once.  Calls one after another: 8191 rows of 96 heads of 128, fp16, 403 MB in
// 78 us, 5.2 TB/s; fp32, 805 MB in 161, 5.0; 16000 rows of 80 heads of 128, three axes, bf16, 656 MB in 122, 5.4 (copies of 200 to 500 MiB: 5.3 to
// 5.4).  Each kernel by itself, as a trace has them: 85 and 132 us for the 16-bit ones.  8 rows 5.8 us in a graph, the rotary store alone 3.5:
// latency, the sum's exchanges and behind them the weights' load.
#pragma once
#include "rope_store_kernel.h"

namespace deinfer {

constexpr int ROPE_MAX_AXES = 4;
constexpr int NORM_MAX_DIM = 2048;               // elements of a head

struct NormRopeParams {
  RopeStoreParams r;
  const void *q_weight, *k_weight;               // [head_dim], or NULL: that side is not normed
  const uint8_t *axis_of;                        // [rot_dim / 2], or NULL: axis 0
  long long pos_pitch;
  double eps;
  int n_axes;
  int lanes;                                     // of a head: a power of two, at most 64
};

// VE consecutive elements as fp32 in one load of 16, 8, 4 or 2 bytes (!WHOLE: one by one, where rows lie at odd elements)
template <typename TE, int VE, bool WHOLE> struct Elems {
  float x[VE];
  __device__ __forceinline__ void load(const TE *p) {
    constexpr int DT = DtOf<TE>::value, B = WHOLE ? VE * (int)sizeof(TE) : 0;
    if constexpr (B == 16) {
      Piece<TE, VE> t;
      t.load(p);
#pragma unroll
      for (int i = 0; i < VE; ++i) x[i] = t.x[i];
    } else if constexpr (sizeof(TE) == 2 && B == 8) {
      const uint2 v = *reinterpret_cast<const uint2 *>(p);
      x[0] = lo_f32<DT>(v.x); x[1] = hi_f32<DT>(v.x); x[2] = lo_f32<DT>(v.y); x[3] = hi_f32<DT>(v.y);
    } else if constexpr (sizeof(TE) == 2 && B == 4) {
      const uint32_t v = *reinterpret_cast<const uint32_t *>(p);
      x[0] = lo_f32<DT>(v); x[1] = hi_f32<DT>(v);
    } else if constexpr (B == 8) {
      const float2 v = *reinterpret_cast<const float2 *>(p);
      x[0] = v.x; x[1] = v.y;
    } else {
#pragma unroll
      for (int i = 0; i < VE; ++i) x[i] = Elem<TE>::load(p + i);
    }
  }
  __device__ __forceinline__ void store(TE *p) const {
    constexpr int DT = DtOf<TE>::value, B = WHOLE ? VE * (int)sizeof(TE) : 0;
    if constexpr (B == 16) {
      Piece<TE, VE> t;
#pragma unroll
      for (int i = 0; i < VE; ++i) t.x[i] = x[i];
      t.store(p);
    } else if constexpr (sizeof(TE) == 2 && B == 8) {
      *reinterpret_cast<uint2 *>(p) = make_uint2(pack2<DT>(x[0], x[1]), pack2<DT>(x[2], x[3]));
    } else if constexpr (sizeof(TE) == 2 && B == 4) {
      *reinterpret_cast<uint32_t *>(p) = pack2<DT>(x[0], x[1]);
    } else if constexpr (B == 8) {
      *reinterpret_cast<float2 *>(p) = make_float2(x[0], x[1]);
    } else {
#pragma unroll
      for (int i = 0; i < VE; ++i) Elem<TE>::store(p + i, x[i]);
    }
  }
  static __device__ __forceinline__ void copy(const TE *p, TE *to) {            // the bits as they are
    constexpr int B = WHOLE ? VE * (int)sizeof(TE) : 0;
    if constexpr (B == 16) *reinterpret_cast<u32x4_t *>(to) = *reinterpret_cast<const u32x4_t *>(p);
    else if constexpr (B == 8) *reinterpret_cast<uint2 *>(to) = *reinterpret_cast<const uint2 *>(p);
    else if constexpr (B == 4) *reinterpret_cast<uint32_t *>(to) = *reinterpret_cast<const uint32_t *>(p);
    else
#pragma unroll
      for (int i = 0; i < VE; ++i) to[i] = p[i];
  }
};

// What a head's elements are multiplied by, from the sum of their squares over the lanes of the head: 1 / sqrt(mean + eps).  Where the
// fp32 sum is out of its comfortable range (elements of 1e19 and more, or all tiny: there an eps that fp32 has no bits for counts too)
// the factor comes from a sum in 64 bits.
struct HeadScale {
  float f;
  double d;
  bool wide;
  __device__ __forceinline__ float of(float x) const { return wide ? (float)((double)x * d) : x * f; }
};
template <typename V> __device__ __forceinline__ V lanes_sum(V x, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}

// VE: elements of one load (2 at least where pairs are interleaved)
template <typename TE, int VE, bool INTER, bool WHOLE>
__global__ __launch_bounds__(ROPE_THREADS) void norm_rope_store_kernel(const NormRopeParams Q) {
  const RopeStoreParams &P = Q.r;
  __shared__ float cs[ROPE_MAX_PAIRS], sn[ROPE_MAX_PAIRS];
  const int t = (int)blockIdx.y * ROPE_GRID + (int)blockIdx.x, tid = threadIdx.x;
  if (t >= P.T) return;
  long long to = t;
  if (P.slots) {
    to = P.slots[t];
    if (to < 0 || to >= P.n_slots) return;                     // a row without a slot is not in use
  }
  const int half = P.rot_dim / 2, D = P.head_dim;
  for (int i = tid; i < half; i += ROPE_THREADS) {
    int axis = Q.axis_of ? Q.axis_of[i] : 0;
    axis = axis < Q.n_axes ? axis : 0;
    float c, s;
    angle_cos_sin(P.positions[axis * Q.pos_pitch + t], P.freqs[i], c, s);
    cs[i] = c * P.magnitude; sn[i] = s * P.magnitude;
  }
  __syncthreads();
  // pieces of one head: rotated ones (in the half layout one piece stands for both of its elements' places), then the others
  const int turned = INTER ? P.rot_dim / VE : half / VE;
  const int pieces = turned + (D - P.rot_dim) / VE;
  const int lanes = Q.lanes, hstep = ROPE_THREADS / lanes, lane = tid & (lanes - 1);
  const int heads = P.n_q + P.n_kv + P.n_v;
  const int second = INTER ? 0 : half;                         // from a rotated piece to its second elements
  for (int hh = tid / lanes; hh < heads; hh += hstep) {        // (the same in the lanes of a head)
    const TE *x, *weight = nullptr;
    TE *y;
    if (hh < P.n_q) {
      x = static_cast<const TE *>(P.q) + t * P.ldq + (long long)hh * D;
      y = static_cast<TE *>(P.q_out) + t * P.ldqo + (long long)hh * D;
      weight = static_cast<const TE *>(Q.q_weight);
    } else if (hh < P.n_q + P.n_kv) {
      const long long h = hh - P.n_q;
      x = static_cast<const TE *>(P.k) + t * P.ldk + h * D;
      y = static_cast<TE *>(P.k_out) + to * P.ldko + h * D;
      weight = static_cast<const TE *>(Q.k_weight);
    } else {
      const long long h = hh - P.n_q - P.n_kv;
      x = static_cast<const TE *>(P.v) + t * P.ldv + h * D;
      y = static_cast<TE *>(P.v_out) + to * P.ldvo + h * D;
      for (int c = lane; c < pieces; c += lanes) {
        const int d = c < turned ? c * VE : P.rot_dim + (c - turned) * VE;
        Elems<TE, VE, WHOLE>::copy(x + d, y + d);
        if (!INTER && c < turned) Elems<TE, VE, WHOLE>::copy(x + d + half, y + d + half);
      }
      continue;
    }
    // a lane's first piece stays in registers; heads of more pieces than lanes read the others again
    Elems<TE, VE, WHOLE> a, b;
#pragma unroll
    for (int e = 0; e < VE; ++e) a.x[e] = b.x[e] = 0.0f;
    auto fetch = [&](int c) {
      const int d = c < turned ? c * VE : P.rot_dim + (c - turned) * VE;
      a.load(x + d);
      if (!INTER) {
        if (c < turned) b.load(x + d + second);
        else
#pragma unroll
          for (int e = 0; e < VE; ++e) b.x[e] = 0.0f;
      }
    };
    if (lane < pieces) fetch(lane);
    HeadScale scale = {1.0f, 1.0, false};
    if (weight) {
      float sum = 0.0f;
      auto squares = [&](float s) {
#pragma unroll
        for (int e = 0; e < VE; ++e) s = fmaf(a.x[e], a.x[e], s);
        if (!INTER)
#pragma unroll
          for (int e = 0; e < VE; ++e) s = fmaf(b.x[e], b.x[e], s);
        return s;
      };
      sum = squares(sum);
      for (int c = lane + lanes; c < pieces; c += lanes) { fetch(c); sum = squares(sum); }
      sum = lanes_sum(sum, lanes);
      const float mean = sum / (float)D + (float)Q.eps;
      scale.wide = !(sum > 1e-30f && sum < 1e38f && mean < 1e38f);
      if (scale.wide) {
        double wide = 0.0;
        for (int c = lane; c < pieces; c += lanes) {
          fetch(c);
#pragma unroll
          for (int e = 0; e < VE; ++e) wide += (double)a.x[e] * a.x[e] + (INTER ? 0.0 : (double)b.x[e] * b.x[e]);
        }
        scale.d = 1.0 / sqrt(lanes_sum(wide, lanes) / D + Q.eps);
      } else {
        scale.f = rsqrtf(mean);
      }
      if (pieces > lanes || scale.wide) {
        if (lane < pieces) fetch(lane);
      }
    }
    for (int c = lane; c < pieces; c += lanes) {
      if (c != lane) fetch(c);
      const int d = c < turned ? c * VE : P.rot_dim + (c - turned) * VE;
      if (weight) {
        Elems<TE, VE, WHOLE> w;
        w.load(weight + d);
#pragma unroll
        for (int e = 0; e < VE; ++e) a.x[e] = scale.of(a.x[e]) * w.x[e];
        if (!INTER && c < turned) {
          w.load(weight + d + second);
#pragma unroll
          for (int e = 0; e < VE; ++e) b.x[e] = scale.of(b.x[e]) * w.x[e];
        }
      }
      if (c < turned) {
        if constexpr (INTER) {
#pragma unroll
          for (int e = 0; e + 1 < VE; e += 2) {
            const float u = a.x[e], w = a.x[e + 1], co = cs[(d + e) / 2], si = sn[(d + e) / 2];
            a.x[e] = u * co - w * si;
            a.x[e + 1] = w * co + u * si;
          }
        } else {
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            const float u = a.x[e], w = b.x[e], co = cs[d + e], si = sn[d + e];
            a.x[e] = u * co - w * si;
            b.x[e] = w * co + u * si;
          }
          b.store(y + d + second);
        }
      }
      a.store(y + d);
    }
  }
}

}  // namespace deinfer
