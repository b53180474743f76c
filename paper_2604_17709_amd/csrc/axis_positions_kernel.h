// Positions of several axes for requests that mix text with images and video.
//
// A request is a list of segments {t, h, w, step}: text of t tokens (h or w not positive), or a grid of t x h x w tokens, row by
// row, frame by frame.  With p the position that a segment begins at, text token i stands at p + i on every axis, and
// grid token (a, b, c) at (p + step a, p + b, p + c); the next segment begins behind the largest of these.  Tokens behind the
// last segment are text.  Whole-number work, bound by the latency of one launch: lengths, segments, two prefix sums, a
// bisection in LDS, stores.  8 requests with a token each 4.0 us, 256 of up to 2000 tokens 7.2 us.  The workgroups of a
// sequence go by the mean length: 131072 tokens alone 7.2 us, beside 255 single ones, by three workgroups, 50.
#pragma once
#include "common.h"

namespace deinfer {

constexpr int PLACE_THREADS = 256;

struct AxisPositionsParams {
  const int4 *segments;
  const int *segment_start, *row_start, *cached;
  int *positions;
  long long pitch;
  int n_segments, n_seqs, T;
};

// Tokens and positions of a segment count up to here: no row's token lies that far on, and positions end at 2^31 - 1.
constexpr long long PLACE_MOST = 1LL << 32;
__device__ __forceinline__ int held_int(long long x) { return x > 0x7fffffffLL ? 0x7fffffff : (int)x; }

// Workgroup (x, y): the sequences x, x + gridDim.x, ..., of each every gridDim.y-th run of PLACE_THREADS rows.
// Segments are taken PLACE_THREADS at a time.
__global__ __launch_bounds__(PLACE_THREADS) void axis_positions_kernel(const AxisPositionsParams P) {
  __shared__ long long token_end[PLACE_THREADS], place_end[PLACE_THREADS];       // sums up to and with each of the present segments
  __shared__ int4 shape[PLACE_THREADS];
  __shared__ long long sums[2][PLACE_THREADS / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int s = blockIdx.x; s < P.n_seqs; s += gridDim.x) {
    int r0 = P.row_start[s], r1 = P.row_start[s + 1], g0 = P.segment_start[s], g1 = P.segment_start[s + 1];
    const long long done = P.cached && P.cached[s] > 0 ? P.cached[s] : 0;
    r0 = r0 < 0 ? 0 : r0; r1 = r1 > P.T ? P.T : r1;
    g0 = g0 < 0 ? 0 : g0; g1 = g1 > P.n_segments ? P.n_segments : g1;
    const int n = r1 > r0 ? r1 - r0 : 0;
    if (n <= (int)blockIdx.y * PLACE_THREADS) continue;          // (the same in every thread)
    long long tokens = 0, place = 0;             // of the segments so far
    // rows [from, to) of the sequence among the workgroup's
    auto rows = [&](long long from, long long to, auto at) {
      from = from < 0 ? 0 : from; to = to > n ? n : to;
      if (from >= to) return;
      const long long step = (long long)gridDim.y * PLACE_THREADS;
      long long i = (from / step) * step + (long long)blockIdx.y * PLACE_THREADS + tid;
      for (; i < to; i += step) {
        if (i < from) continue;
        int a, b, c;
        at(i + done, a, b, c);
        int *p = P.positions + r0 + i;
        p[0] = a; p[P.pitch] = b; p[2 * P.pitch] = c;
      }
    };
    for (int g = g0; g < g1; g += PLACE_THREADS) {
      int4 e = make_int4(0, 0, 0, 0);
      if (g + tid < g1) e = P.segments[g + tid];
      const bool text = e.y <= 0 || e.z <= 0;
      long long count = e.x > 0 ? e.x : 0, ahead = count;
      if (!text && count > 0) {
        const long long hw = (long long)e.y * e.z, far = (long long)(e.w > 0 ? e.w : 0) * (count - 1);
        ahead = (far > e.y - 1 ? far : e.y - 1);
        ahead = (ahead > e.z - 1 ? ahead : e.z - 1) + 1;
        count *= hw > PLACE_MOST ? PLACE_MOST : hw;          // (below 2^63)
      }
      long long ct = count > PLACE_MOST ? PLACE_MOST : count, ca = ahead > PLACE_MOST ? PLACE_MOST : ahead;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const long long u = __shfl_up(ct, o, 64), v = __shfl_up(ca, o, 64);
        if (lane >= o) { ct += u; ca += v; }
      }
      __syncthreads();                           // (the segments before are read)
      if (lane == 63) { sums[0][wave] = ct; sums[1][wave] = ca; }
      __syncthreads();
      long long all_t = 0, all_a = 0;
      for (int w = 0; w < PLACE_THREADS / 64; ++w) {
        if (w < wave) { ct += sums[0][w]; ca += sums[1][w]; }
        all_t += sums[0][w]; all_a += sums[1][w];
      }
      token_end[tid] = tokens + ct; place_end[tid] = place + ca;
      shape[tid] = e;
      __syncthreads();
      const int most = g1 - g < PLACE_THREADS ? g1 - g : PLACE_THREADS;
      rows(tokens - done, tokens + all_t - done, [&](long long token, int &a, int &b, int &c) {
        int lo = 0, hi = most - 1;               // the first segment that ends behind the token
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (token_end[mid] > token) hi = mid; else lo = mid + 1;
        }
        const long long r = token - (lo ? token_end[lo - 1] : tokens), p = lo ? place_end[lo - 1] : place;
        const int4 e = shape[lo];
        if (e.y <= 0 || e.z <= 0) {
          a = b = c = held_int(p + r);
        } else {
          const long long hw = (long long)e.y * e.z;
          const uint32_t frame = hw > r ? 0u : (uint32_t)r / (uint32_t)hw, in = (uint32_t)(r - frame * hw), line = in / (uint32_t)e.z;
          a = held_int(p + (long long)frame * (e.w > 0 ? e.w : 0)); b = held_int(p + line); c = held_int(p + (in - line * (uint32_t)e.z));
        }
      });
      tokens += all_t; place += all_a;
    }
    rows(tokens - done, (long long)n, [&](long long token, int &a, int &b, int &c) { a = b = c = held_int(place + token - tokens); });
    __syncthreads();                             // (before the next sequence's segments)
  }
}

}  // namespace deinfer
