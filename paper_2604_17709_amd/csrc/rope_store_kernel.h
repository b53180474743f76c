// Rotary positions on the way into the paged cache: queries rotated, keys rotated into their slots,
// values stored beside them, in one pass.
//
//   a = positions[t] * freqs[i]        (the angle of pair i, i < rot_dim / 2)
//   x_first  <- m (x_first cos a - x_second sin a)
//   x_second <- m (x_second cos a + x_first sin a)
//
// with the pair (i, i + rot_dim / 2) of a head, or (2 i, 2 i + 1) where pairs are interleaved; elements from
// rot_dim on, and values, are copied.  Bound by HBM: every element is read once and written once.  A workgroup takes
// one token: its threads first form the token's cosines and sines once, in LDS, and then
// go over the heads with 16-byte loads and stores, so the angles cost 1 / heads of what forming them per head would.
// 8191 tokens, 32 + 32 + 32 heads of 128: 78 us for 402 MB = 5.1 TB/s, what a large copy reaches; 8 tokens: 4.1 us.
#pragma once
#include "common.h"

namespace deinfer {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_MAX_PAIRS = 512;
constexpr int ROPE_GRID = 1 << 20;               // tokens of one row of the grid: its threads have to stay below 2^32

struct RopeStoreParams {
  const void *q, *k, *v;
  void *q_out, *k_out, *v_out;
  const int *positions, *slots;
  const double *freqs;
  long long ldq, ldk, ldv, ldqo, ldko, ldvo, n_slots;
  int T, n_q, n_kv, n_v, head_dim, rot_dim;                    // n_q, n_kv, n_v: heads of q, k, v (0: not given)
  float magnitude;
};

// cosine and sine of an angle that may be 1e9 radians: the revolutions in double precision, their fraction
// (2^-25 at most off) in single
__device__ __forceinline__ void angle_cos_sin(int pos, double freq, float &c, float &s) {
  const double rev = (double)pos * freq * 0.15915494309189535;        // 1 / (2 pi)
  sincospif(2.0f * (float)(rev - rint(rev)), &s, &c);
}

// VE consecutive elements as fp32
template <typename TE, int VE> struct Piece {
  float x[VE];
  __device__ __forceinline__ void load(const TE *p) {
    if constexpr (VE * sizeof(TE) == 16 && sizeof(TE) == 2) {
      constexpr int DT = DtOf<TE>::value;
      const u32x4_t v = *reinterpret_cast<const u32x4_t *>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) { x[2 * i] = lo_f32<DT>(v[i]); x[2 * i + 1] = hi_f32<DT>(v[i]); }
    } else if constexpr (VE * sizeof(TE) == 16) {
      const f32x4_t v = *reinterpret_cast<const f32x4_t *>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = v[i];
    } else {
#pragma unroll
      for (int i = 0; i < VE; ++i) x[i] = Elem<TE>::load(p + i);
    }
  }
  static __device__ __forceinline__ void copy(const TE *p, TE *to) {            // the bits as they are
    if constexpr (VE * sizeof(TE) == 16) {
      *reinterpret_cast<u32x4_t *>(to) = *reinterpret_cast<const u32x4_t *>(p);
    } else {
#pragma unroll
      for (int i = 0; i < VE; ++i) to[i] = p[i];
    }
  }
  __device__ __forceinline__ void store(TE *p) const {
    if constexpr (VE * sizeof(TE) == 16 && sizeof(TE) == 2) {
      constexpr int DT = DtOf<TE>::value;
      u32x4_t v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = pack2<DT>(x[2 * i], x[2 * i + 1]);
      *reinterpret_cast<u32x4_t *>(p) = v;
    } else if constexpr (VE * sizeof(TE) == 16) {
      *reinterpret_cast<f32x4_t *>(p) = f32x4_t{x[0], x[1], x[2], x[3]};
    } else {
#pragma unroll
      for (int i = 0; i < VE; ++i) Elem<TE>::store(p + i, x[i]);
    }
  }
};

// VE: elements of one load; 16 bytes, or where rows, heads or the rotated part are not made of 16-byte pieces 1
// (2 for interleaved pairs)
template <typename TE, int VE, bool INTER>
__global__ __launch_bounds__(ROPE_THREADS) void rope_store_kernel(const RopeStoreParams P) {
  __shared__ float cs[ROPE_MAX_PAIRS], sn[ROPE_MAX_PAIRS];
  const int t = (int)blockIdx.y * ROPE_GRID + (int)blockIdx.x, tid = threadIdx.x;
  if (t >= P.T) return;
  long long to = t;
  if (P.slots) {
    to = P.slots[t];
    if (to < 0 || to >= P.n_slots) return;                     // a row without a slot is not in use
  }
  const int half = P.rot_dim / 2, D = P.head_dim;
  if (half > 0) {
    const int pos = P.positions[t];
    for (int i = tid; i < half; i += ROPE_THREADS) {
      float c, s;
      angle_cos_sin(pos, P.freqs[i], c, s);
      cs[i] = c * P.magnitude; sn[i] = s * P.magnitude;
    }
    __syncthreads();
  }
  // pieces of one head: rotated ones (in the half layout one piece stands for both of its elements' places), then copied ones
  const int turned = INTER ? P.rot_dim / VE : half / VE;
  const int pieces = turned + (D - P.rot_dim) / VE;
  const int lanes = pieces < ROPE_THREADS ? pieces : ROPE_THREADS, hstep = ROPE_THREADS / lanes;
  const int heads = P.n_q + P.n_kv + P.n_v;
  if (tid >= lanes * hstep) return;
  for (int hh = tid / lanes; hh < heads; hh += hstep) {
    const TE *x;
    TE *y;
    bool rotate = true;
    if (hh < P.n_q) {
      x = static_cast<const TE *>(P.q) + t * P.ldq + (long long)hh * D;
      y = static_cast<TE *>(P.q_out) + t * P.ldqo + (long long)hh * D;
    } else if (hh < P.n_q + P.n_kv) {
      const long long h = hh - P.n_q;
      x = static_cast<const TE *>(P.k) + t * P.ldk + h * D;
      y = static_cast<TE *>(P.k_out) + to * P.ldko + h * D;
    } else {
      const long long h = hh - P.n_q - P.n_kv;
      x = static_cast<const TE *>(P.v) + t * P.ldv + h * D;
      y = static_cast<TE *>(P.v_out) + to * P.ldvo + h * D;
      rotate = false;
    }
    for (int c = tid % lanes; c < pieces; c += lanes) {
      const int d = c < turned ? c * VE : P.rot_dim + (c - turned) * VE;
      if (!rotate || c >= turned) {
        Piece<TE, VE>::copy(x + d, y + d);
        if (!INTER && c < turned) Piece<TE, VE>::copy(x + d + half, y + d + half);
      } else if constexpr (INTER) {
        Piece<TE, VE> a;
        a.load(x + d);
#pragma unroll
        for (int e = 0; e + 1 < VE; e += 2) {
          const float u = a.x[e], w = a.x[e + 1], co = cs[(d + e) / 2], si = sn[(d + e) / 2];
          a.x[e] = u * co - w * si;
          a.x[e + 1] = w * co + u * si;
        }
        a.store(y + d);
      } else {
        Piece<TE, VE> a, b;
        a.load(x + d);
        b.load(x + d + half);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const float u = a.x[e], w = b.x[e], co = cs[d + e], si = sn[d + e];
          a.x[e] = u * co - w * si;
          b.x[e] = w * co + u * si;
        }
        a.store(y + d);
        b.store(y + d + half);
      }
    }
  }
}

}  // namespace deinfer
