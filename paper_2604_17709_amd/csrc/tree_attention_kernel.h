// Attention of a step's tokens (one per sequence, a drafted tree, a chunk of a prompt) over a paged cache.
//
// For a row (token i of sequence s, query head h) and the keys it sees, all c cached tokens of s and
// those of the step's own tokens that its mask names,
//   o = sum_t exp(x_t - max x) v_t / sum_t exp(x_t - max x),   x_t = scale q . k_t,
// in one pass over the keys: running maximum m, running sum l and unnormalised output O per row, all in
// fp32; a new maximum multiplies l and O by exp(m_old - m_new).
//
// A wavefront holds tiles of 16 rows and goes through the keys 32 at a time.  The first product is formed
// transposed, S^T = K Q^T, so that a lane has the scores of ONE row (l % 16) and of eight keys: the softmax's
// reductions are in-lane but for two steps across the wave's quarters, and the eight probabilities are, as
// they stand, the lane's share of the second product's operand P^T if its k index is read as
//   8 (l / 16) + 4 u + i  <->  key 16 u + 4 (l / 16) + i,   u < 2, i < 4.
// The other operand V^T needs, per lane, eight keys of one feature.  A lane loads 8 neighbouring features of
// those eight keys (a quarter wave reads whole rows of V) and swaps the 16-bit halves of its own registers:
// 32 byte-permutes turn the 8 x 8 block into eight operands, one for every 8th feature.  Neither P nor V
// crosses lanes, and neither product needs LDS.
//
// Work is counted in units (UNIT keys of one tile of rows), over all sequences, key heads and row tiles, and
// every workgroup takes an equal run of units, wherever sequences begin and end: ragged lengths, few long
// sequences and many short ones all fill the device.  The run is found on the device from the lengths, so one
// captured launch serves every later step.  A tile of rows whose keys several workgroups share leaves partial
// (O, m, l) in the workspace, at most two per workgroup, and a second launch joins them in order; results do
// not depend on timing.
#pragma once
#include "common.h"

namespace deinfer {

constexpr int ATT_THREADS = 256;
constexpr int ATT_KEYS = 32;                     // keys of one step of a wavefront

struct AttParams {
  const uint16_t *q, *k, *v;
  uint16_t *out;
  const int *row_start, *cached, *table;
  const uint32_t *mask;
  long long ldq, ldo;
  uint32_t ldk, ldv;                             // in bytes
  int table_pitch, n_pool_blocks, most_keys;     // most_keys: tokens that a row of the table can hold, at most 2^30
  int T, n_seqs, n_kv, group, head_dim, block_tokens, block_shift, mask_words;
  float scale2;                                  // scale log2(e): the exponentials are powers of two
  int n_shares;
  float *part;                                   // [2 n_shares][rows][DP] partial outputs
  float2 *part_ml;                               // [2 n_shares][rows] their maxima and sums
  int4 *joins;                                   // [n_shares] tile of rows whose first share this is and that others share (sequence, head, tile, shares)
};

struct AttSeq { int row0, n, ctx, keys; };       // first row, rows, cached tokens, keys in all
__device__ __forceinline__ AttSeq att_seq(const AttParams &P, int s) {
  AttSeq q;
  int r0 = P.row_start[s], r1 = P.row_start[s + 1];
  r0 = r0 < 0 ? 0 : r0; r1 = r1 > P.T ? P.T : r1;
  q.row0 = r0; q.n = r1 > r0 ? r1 - r0 : 0;
  const int c = P.cached[s];
  q.ctx = c < 0 ? 0 : c < P.most_keys ? c : P.most_keys;          // (what the table has no room for is not seen)
  q.keys = q.n < P.most_keys - q.ctx ? q.ctx + q.n : P.most_keys;
  return q;
}
// a value that is the same in every lane, in scalar registers
__device__ __forceinline__ long long uniform(long long x) {
  return ((long long)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x);
}
// Keys that some row of a tile sees: all of the sequence's, or in a causal chunk none behind the tile's last token.
template <int ROWS> __device__ __forceinline__ int att_tile_keys(const AttParams &P, const AttSeq &q, int tile) {
  const int rows = q.n * P.group, end = (tile + 1) * ROWS < rows ? (tile + 1) * ROWS : rows;
  const int causal = q.ctx + (end - 1) / P.group + 1;             // (at most 2^30 + 2^28)
  return P.mask || causal > q.keys ? q.keys : causal;
}
template <int ROWS, int UNIT> __device__ __forceinline__ int att_tile_units(const AttParams &P, const AttSeq &q, int tile) {
  const int u = (att_tile_keys<ROWS>(P, q, tile) + UNIT - 1) / UNIT;
  return u < 1 ? 1 : u;                          // (rows without any key are written too)
}
// A tile costs a workgroup START units' time before and after its units, which are counted, so that many short tiles are
// spread as evenly as a few long ones: START units of nobody's lie ahead of each tile's.  16 sequences of 1 to 16k keys
// with 64 drafted tokens: 539 us without, 441 with 6, 451 with 20; 64 sequences of up to 8k with one row: 217, 218 with 1,
// 221 with 2.
template <int ROWS> constexpr int ATT_START = ROWS == 16 ? 1 : 8;
// units of one key head of a sequence
template <int ROWS, int UNIT> __device__ __forceinline__ long long att_head_units(const AttParams &P, const AttSeq &q) {
  constexpr int START = ATT_START<ROWS>;
  const int tiles = (q.n * P.group + ROWS - 1) / ROWS;
  if (P.mask || tiles <= 1) return tiles ? (long long)tiles * (START + att_tile_units<ROWS, UNIT>(P, q, tiles - 1)) : 0;
  long long u = 0;
  for (int t = 0; t < tiles; ++t) u += START + att_tile_units<ROWS, UNIT>(P, q, t);
  return u;
}

// A workgroup's run of units, tile after tile.  Everything is the same in all lanes.
template <int ROWS, int UNIT, int THREADS> struct AttRun {
  static constexpr int START = ATT_START<ROWS>;
  long long per_share, cur, end, base;           // base: first unit of the present tile (behind its START)
  AttSeq seq;
  int s, h, tile, per_tile;

  // scan: THREADS / 64 values, found: 2 values of LDS.  False: nothing to do
  __device__ __forceinline__ bool begin(const AttParams &P, int share, long long *scan, long long *found) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    auto units_of = [&](int x) -> long long { return x < P.n_seqs ? P.n_kv * att_head_units<ROWS, UNIT>(P, att_seq(P, x)) : 0; };
    auto scan_units = [&](long long u, long long *total) {           // inclusive sum over the threads
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const long long w = __shfl_up(u, o, 64);
        if (lane >= o) u += w;
      }
      __syncthreads();
      if (lane == 63) scan[wave] = u;
      __syncthreads();
      long long all = 0, before = 0;
      for (int w = 0; w < THREADS / 64; ++w) { if (w < wave) before += scan[w]; all += scan[w]; }
      *total = all;
      return u + before;
    };
    // (the last pass over up to THREADS sequences is kept: with no more of them there is one pass)
    long long total = 0, mine = 0, mine_end = 0;
    for (int s0 = 0; s0 < P.n_seqs; s0 += THREADS) {
      long long t;
      mine = units_of(s0 + tid);
      mine_end = scan_units(mine, &t);
      total += t;
    }
    total = uniform(total);
    per_share = (total + P.n_shares - 1) / P.n_shares;
    cur = per_share * share;
    end = cur + per_share < total ? cur + per_share : total;
    if (cur >= end) return false;
    long long before = 0;
    for (int s0 = 0; s0 < P.n_seqs; s0 += THREADS) {
      long long t = total;
      if (P.n_seqs > THREADS) {
        mine = units_of(s0 + tid);
        mine_end = scan_units(mine, &t);
      }
      const long long e = before + mine_end;
      if (mine > 0 && e - mine <= cur && cur < e) { found[0] = s0 + tid; found[1] = e - mine; }
      before += t;
      if (before > cur) break;
    }
    __syncthreads();
    s = __builtin_amdgcn_readfirstlane((int)found[0]);
    base = uniform(found[1]);
    seq = att_seq(P, s);
    const long long per_head = uniform(att_head_units<ROWS, UNIT>(P, seq));
    h = (int)((cur - base) / per_head);
    base += h * per_head + START;
    tile = 0;
    per_tile = att_tile_units<ROWS, UNIT>(P, seq, 0);
    while (cur >= base + per_tile) { base += per_tile + START; per_tile = att_tile_units<ROWS, UNIT>(P, seq, ++tile); }
    if (cur < base) cur = base;
    return cur < end;
  }
  // The present tile's units [from, to); then on to the next tile.
  __device__ __forceinline__ int from() const { return (int)(cur - base); }
  __device__ __forceinline__ int to() const { return end - base < per_tile ? (int)(end - base) : per_tile; }
  __device__ __forceinline__ bool next(const AttParams &P) {
    base += per_tile + START;
    if (base >= end) return false;
    cur = base;
    if ((tile + 1) * ROWS < seq.n * P.group) {
      ++tile;
    } else {
      tile = 0;
      if (++h == P.n_kv) {
        h = 0;
        do { seq = att_seq(P, ++s); } while (seq.n == 0 && s + 1 < P.n_seqs);
      }
    }
    per_tile = att_tile_units<ROWS, UNIT>(P, seq, tile);
    return true;
  }
  // shares that have units of the present tile
  __device__ __forceinline__ int sharers() const { return (int)((base + per_tile - 1) / per_share - base / per_share + 1); }
};

__device__ __forceinline__ float att_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
// the largest of the four quarters of the wave, in every lane
__device__ __forceinline__ float quarters_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16, 64));
  return fmaxf(x, __shfl_xor(x, 32, 64));
}

// Bits of the 32 keys from k0 on that row `token` of the sequence sees among the drafted ones (all ones for cached keys).
__device__ __forceinline__ uint32_t att_window(const AttParams &P, const AttSeq &q, int k0, int token, bool row) {
  if (!P.mask) {
    const int n = q.ctx + token + 1 - k0;
    return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u;
  }
  const int e = k0 - q.ctx;                      // first of the 32 as index among the step's own tokens
  if (e <= -32) return 0xffffffffu;
  const uint32_t *mw = P.mask + (long long)(q.row0 + token) * P.mask_words;
  auto word = [&](int i) -> uint32_t { return row && i < P.mask_words ? mw[i] : 0u; };
  if (e < 0) return (word(0) << -e) | ((1u << -e) - 1u);
  uint32_t w = word(e >> 5) >> (e & 31);
  if (e & 31) w |= word((e >> 5) + 1) << (32 - (e & 31));
  return w;
}

// 16-bit elements of a word that are infinite or NaN
template <int DT> __device__ __forceinline__ bool not_finite(uint32_t w) {
  constexpr uint32_t E = DT == DT_F16 ? 0x7c00u : 0x7f80u;
  return (w & E) == E || (w & (E << 16)) == (E << 16);
}

// DP: head dimension up to 64, 128 or 256; FULL: it is DP; POW2: blocks of a power of two of at least 16
// tokens (16 neighbouring keys are rows of one block: their address is one scalar and a lane's constant);
// one tile of 16 rows, over four wavefronts' interleaved shares of the keys, which are merged in LDS.
// Bound by reading the cache: 64 sequences of up to 8191 cached tokens, 8 key heads of 128, one token each: 217 us for 1.13 GB =
// 5.2 TB/s (a read alone: 6.0); three workgroups per unit in fewer registers: 225, four: 266.  8 sequences of up to 1000: 11.5 us,
// which is one dependent chain: lengths, block ids, rows, merge.
template <int DT, int DP, bool FULL, bool POW2>
__global__ __launch_bounds__(ATT_THREADS) void tree_attention_kernel(const AttParams P) {
  constexpr int WK = ATT_THREADS / 64, ROWS = 16, UNIT = ATT_KEYS * WK;
  constexpr int KS = DP / 32;                    // k steps of the first product
  constexpr int VE = DP == 64 ? 4 : 8;           // neighbouring features of V per lane and piece
  constexpr int NC = DP / (16 * VE);             // pieces
  constexpr int NF = NC * VE;                    // 16-feature blocks of the output
  constexpr int VW = VE / 2;                     // words of a piece
  constexpr int OP = DP + 4;                     // row pitch of the merge buffer in LDS
  // The largest probability of a row: fp16's smallest normal number is 2^-14, and what lies below it has fewer bits and is
  // nothing from 2^-25 on, which a long tail of keys may add up to a good part of the output.  O and l have the factor alike.
  constexpr float LIFT = DT == DT_F16 ? 32768.0f : 1.0f;
  constexpr uint32_t ONES = DT == DT_F16 ? 0x3c003c00u : 0x3f803f80u;
  __shared__ __attribute__((aligned(16))) float merge_o[WK * 16 * OP];
  __shared__ float merge_ml[2 * WK * 16];
  __shared__ long long scan[ATT_THREADS / 64];
  __shared__ long long found[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, quarter = lane >> 4;
  const int D = FULL ? DP : P.head_dim;
  const int share = run_tile_of(blockIdx.x, P.n_shares);

  AttRun<ROWS, UNIT, ATT_THREADS> run;
  if (tid == 0) P.joins[share] = make_int4(-1, 0, 0, 0);
  if (!run.begin(P, share, scan, found)) return;                   // (the same in every thread)
  do {
    const AttSeq seq = run.seq;
    const int s = run.s, h = run.h, tile = run.tile, u0 = run.from(), u1 = run.to();

    // ---- the rows
    const int n_rows = seq.n * P.group - tile * ROWS < ROWS ? seq.n * P.group - tile * ROWS : ROWS;   // of this tile
    const int gr = tile * ROWS + col, token = gr / P.group;           // this lane's row
    u32x4_t qf[KS];
    {
      const uint16_t *qp = P.q + (long long)(seq.row0 + token) * P.ldq + (long long)(h * P.group + gr - token * P.group) * D + quarter * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qf[ks] = u32x4_t{0u, 0u, 0u, 0u};
        if (col < n_rows && (FULL || ks * 32 + quarter * 8 < D)) qf[ks] = *reinterpret_cast<const u32x4_t *>(qp + ks * 32);
      }
    }
    f32x4_t o[NF], l = {0.0f, 0.0f, 0.0f, 0.0f};
    float m = -__builtin_inff();
    const u32x4_t ones = {ONES, ONES, ONES, ONES};
#pragma unroll
    for (int f = 0; f < NF; ++f) o[f] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    // keys that some row may see, and keys that every row sees
    const int keys_end = att_tile_keys<ROWS>(P, seq, tile);
    const int keys_all = P.mask ? seq.ctx : seq.ctx + tile * ROWS / P.group + 1;

    const int *table = P.table + (long long)s * P.table_pitch;
    const char *kh = reinterpret_cast<const char *>(P.k + (long long)h * D), *vh = reinterpret_cast<const char *>(P.v + (long long)h * D);
    const uint32_t klane = col * P.ldk + quarter * 16, vlane = quarter * 4 * P.ldv + col * VE * 2;
    const int k_last = u1 * UNIT < keys_end ? u1 * UNIT : keys_end;
    for (int k0 = u0 * UNIT + wave * ATT_KEYS; k0 < k_last; k0 += UNIT) {
      // ---- where the 32 keys are; `live`: those that exist
      uint32_t live = keys_end - k0 >= 32 ? 0xffffffffu : (1u << (keys_end - k0)) - 1u;
      const char *kp[2], *vp[2];                 // POW2: rows of the two halves' first keys
      int slot = 0;                              // otherwise: row of the key k0 + lane % 32
      if constexpr (POW2) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int kk = k0 + 16 * u;
          int id = -1;
          if (kk < keys_end) id = table[kk >> P.block_shift];
          const bool ok = id >= 0 && id < P.n_pool_blocks;
          if (!ok) live &= ~(0xffffu << (16 * u));
          const uint64_t row = ok ? (uint32_t)((id << P.block_shift) + (kk & (P.block_tokens - 1))) : 0u;
          kp[u] = kh + row * P.ldk;
          vp[u] = vh + row * P.ldv;
        }
      } else {
        const int kk = k0 + (lane & 31);
        bool ok = false;
        if (kk < keys_end) {
          const int page = kk / P.block_tokens, id = table[page];
          ok = id >= 0 && id < P.n_pool_blocks;
          if (ok) slot = id * P.block_tokens + (kk - page * P.block_tokens);
        }
        live &= (uint32_t)__ballot(ok);
      }
      u32x4_t kf[2][KS];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const char *kr;
        if constexpr (POW2) kr = kp[u] + klane;
        else kr = kh + (uint64_t)(uint32_t)__shfl(slot, 16 * u + col, 64) * P.ldk + quarter * 16;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          kf[u][ks] = u32x4_t{0u, 0u, 0u, 0u};
          if (FULL || ks * 32 + quarter * 8 < D) kf[u][ks] = *reinterpret_cast<const u32x4_t *>(kr + ks * 64);
        }
      }
      uint32_t vw[NC][8][VW];                    // [piece][key 4 u + i of the lane][word]
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const char *vr;
        if constexpr (POW2) vr = vp[x / 4] + (x % 4) * P.ldv + vlane;
        else vr = vh + (uint64_t)(uint32_t)__shfl(slot, 16 * (x / 4) + 4 * quarter + x % 4, 64) * P.ldv + col * VE * 2;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
#pragma unroll
          for (int w = 0; w < VW; ++w) vw[c][x][w] = 0u;
          if (FULL || c * 16 * VE + col * VE < D) {
            if constexpr (VE == 8) {
              const u32x4_t t = *reinterpret_cast<const u32x4_t *>(vr + c * 256);
#pragma unroll
              for (int w = 0; w < 4; ++w) vw[c][x][w] = t[w];
            } else {
              const uint2 t = *reinterpret_cast<const uint2 *>(vr);
              vw[c][x][0] = t.x; vw[c][x][1] = t.y;
            }
          }
        }
      }
      // ---- what each row sees of the 32 keys
      const bool masked = live != 0xffffffffu || k0 + 32 > keys_all;
      uint32_t sees = 0xffffffffu;
      bool odd_v = false;                        // a value that is infinite or NaN beside rows that do not see it
      if (masked) {
#pragma unroll
        for (int x = 0; x < 8; ++x) {            // rows of V that hold no key: whatever is there counts as zero
          const bool there = (live >> (16 * (x / 4) + 4 * quarter + x % 4)) & 1u;
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int w = 0; w < VW; ++w) {
              if (!there) vw[c][x][w] = 0u;
              odd_v |= not_finite<DT>(vw[c][x][w]);
            }
        }
        odd_v = __any(odd_v);
        sees = att_window(P, seq, k0, token, col < n_rows) & live;
      }
      f32x4_t sc[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        sc[u] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) sc[u] = mfma16<DT>(kf[u][ks], qf[ks], sc[u]);
      }
      float p[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) p[x] = sc[x / 4][x % 4] * P.scale2;
      if (masked) {
#pragma unroll
        for (int x = 0; x < 8; ++x)
          if (!((sees >> (16 * (x / 4) + 4 * quarter + x % 4)) & 1u)) p[x] = -__builtin_inff();
      }
      float top = p[0];
#pragma unroll
      for (int x = 1; x < 8; ++x) top = fmaxf(top, p[x]);
      top = quarters_max(top);
      if (__any(top > m)) {
        const float m_new = fmaxf(m, top);
        const float a = m == -__builtin_inff() ? 0.0f : att_exp2(m - m_new);
        m = m_new;
#pragma unroll
        for (int i = 0; i < 4; ++i) l[i] *= a;
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[f][i] *= a;
      }
      const float base = m == -__builtin_inff() ? 0.0f : m;     // (a row that has seen no key yet)
#pragma unroll
      for (int x = 0; x < 8; ++x) p[x] = att_exp2(p[x] - base) * LIFT;
      // the probabilities, at most LIFT, as the 16-bit operand of the second product: each is off by at most half a
      // step of the type (those of normal size, which reach down to 2^-29 of the largest in fp16), which is what the output's own
      // rounding is off by; the sum is that of the rounded ones
      const u32x4_t pf = {pack2<DT>(p[0], p[1]), pack2<DT>(p[2], p[3]), pack2<DT>(p[4], p[5]), pack2<DT>(p[6], p[7])};
      l = mfma16<DT>(ones, pf, l);
      if (!masked || !odd_v) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            u32x4_t vf;
#pragma unroll
            for (int w = 0; w < 4; ++w)
              vf[w] = __builtin_amdgcn_perm(vw[c][2 * w + 1][e / 2], vw[c][2 * w][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
            o[c * VE + e] = mfma16<DT>(vf, pf, o[c * VE + e]);
          }
      } else {
        // 0 x infinity is no number: with such a value among the keys, every row adds up the keys that it sees, one by one
#pragma unroll 1
        for (int kk = 0; kk < 32; ++kk) {
          if (!((live >> kk) & 1u)) continue;
          const int x0 = 4 * (kk >> 4) + (kk & 3);
          uint32_t w = pf[0];
#pragma unroll
          for (int x = 1; x < 4; ++x) w = (x0 >> 1) == x ? pf[x] : w;
          const float mine = x0 & 1 ? hi_f32<DT>(w) : lo_f32<DT>(w);
          const float pk = __shfl(mine, ((kk >> 2) & 3) * 16 + col, 64);
          const bool see = (sees >> kk) & 1u;
          const uint16_t *vr;
          if constexpr (POW2) vr = reinterpret_cast<const uint16_t *>((kk < 16 ? vp[0] : vp[1]) + (kk & 15) * P.ldv);
          else vr = reinterpret_cast<const uint16_t *>(vh + (uint64_t)(uint32_t)__shfl(slot, kk, 64) * P.ldv);
#pragma unroll
          for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int d = (f / VE) * 16 * VE + (quarter * 4 + i) * VE + f % VE;
              if (see && (FULL || d < D)) o[f][i] += pk * cvt_in<DT>(vr[d]);
            }
        }
      }
    }

    // ---- out: to the rows, where this workgroup had all their keys, else to the workspace
    const bool whole = u0 == 0 && u1 == run.per_tile;
    const long long which = 2LL * share + (u0 == 0 ? 1 : 0);        // (a tile that begins here is the last of the run, one that does not the first)
    auto store_row = [&](int r, int d, const float *x, float mm, float ll) {      // VE features from d of row r of the tile; ll: their sum
      if (whole) {
        const int gr = tile * ROWS + r, j = gr / P.group, hh = gr - j * P.group;
        uint16_t *op = P.out + (long long)(seq.row0 + j) * P.ldo + (long long)(h * P.group + hh) * D + d;
        const float inv = ll > 0.0f || ll != ll ? 1.0f / ll : 0.0f;               // (no key seen: zeros)
        uint32_t w[VW];
#pragma unroll
        for (int i = 0; i < VW; ++i) w[i] = pack2<DT>(x[2 * i] * inv, x[2 * i + 1] * inv);
        if constexpr (VE == 8) *reinterpret_cast<u32x4_t *>(op) = u32x4_t{w[0], w[1], w[2], w[3]};
        else *reinterpret_cast<uint2 *>(op) = make_uint2(w[0], w[1]);
      } else {
        float *pp = P.part + (which * ROWS + r) * DP + d;
#pragma unroll
        for (int i = 0; i < VE; i += 4) *reinterpret_cast<f32x4_t *>(pp + i) = f32x4_t{x[i], x[i + 1], x[i + 2], x[i + 3]};
        if (d == 0) P.part_ml[which * ROWS + r] = make_float2(mm, ll);
      }
    };
    __syncthreads();                                            // (the buffer's last readers are done)
    if (quarter == 0) { merge_ml[(wave * 16 + col) * 2] = m; merge_ml[(wave * 16 + col) * 2 + 1] = l[0]; }
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float *mp = merge_o + (wave * 16 + col) * OP + c * 16 * VE + (quarter * 4 + i) * VE;
#pragma unroll
        for (int e = 0; e < VE; e += 4)
          *reinterpret_cast<f32x4_t *>(mp + e) = f32x4_t{o[c * VE + e][i], o[c * VE + e + 1][i], o[c * VE + e + 2][i], o[c * VE + e + 3][i]};
      }
    __syncthreads();
    for (int x = tid; x < 16 * (DP / VE); x += ATT_THREADS) {
      const int rr = x / (DP / VE), d = (x - rr * (DP / VE)) * VE;
      if (rr >= n_rows || (!FULL && d >= D)) continue;
      float mm = merge_ml[rr * 2], ll = 0.0f, y[VE];
#pragma unroll
      for (int w = 1; w < WK; ++w) mm = fmaxf(mm, merge_ml[(w * 16 + rr) * 2]);
#pragma unroll
      for (int e = 0; e < VE; ++e) y[e] = 0.0f;
#pragma unroll
      for (int w = 0; w < WK; ++w) {
        // (a part without any key has l = 0 and O = 0, or, where all its scores were no numbers, neither: kept as it is)
        const float mw = merge_ml[(w * 16 + rr) * 2], a = mw == -__builtin_inff() ? 1.0f : att_exp2(mw - mm);
        ll += a * merge_ml[(w * 16 + rr) * 2 + 1];
#pragma unroll
        for (int e = 0; e < VE; ++e) y[e] += a * merge_o[(w * 16 + rr) * OP + d + e];
      }
      store_row(rr, d, y, mm, ll);
    }
    if (!whole && u0 == 0 && tid == 0) P.joins[share] = make_int4(s, h, tile, run.sharers());
  } while (run.next(P));
}

// The same work where a sequence and key head has more than a few rows: eight wavefronts with RT tiles of 16 rows each
// share the keys, STAGE at a time, through LDS, a ring of four stages.  The rows of K and V come straight from
// memory into the ring, three stages ahead of their use (no registers, no waiting; one barrier per stage).  Rows
// lie in LDS as they do in memory but for their 16-byte pieces, which are XORed with the row's number.  With heads of 128 and 256
// sixteen rows at one place (an operand of K) then cover all banks; with heads of 64, whose rows are half of the banks
// wide, rows r and r + 8 meet.  The transposing read that makes V^T's operand takes the pieces 2 f and 2 f + 1 of its rows, and the
// XOR only swaps those two between the rows 2 n and 2 n + 1: with heads of 128 it covers half of the banks twice, two cycles of conflict
// per read (SQ_LDS_BANK_CONFLICT: 1.45e7 cycles in 7.3e6 such reads).  V needs no permutes here, and its features keep their
// order: block f of the output is 16 f .. 16 f + 15.
//
// Measured (64 drafted tokens x 16 sequences of up to 16384 keys, 8 key heads of 128, fp16): 339 us a call, about 4200 cycles for
// 64 keys and 256 rows.  2176 of them are matrix instructions (two wavefronts per SIMD); the LDS reads of all eight wavefronts
// are 256 KiB, 2048 cycles at 128 bytes each, and 512 cycles of conflicts.  2 x 2048 prompt tokens on up to 6000 cached, 32 heads,
// bf16: 411 us = 816 TFLOP/s.
// Under such calls the clock falls to its power limit (half of the wavefronts asleep for 640 cycles of every stage cost nothing), so
// fewer instructions count for more than a better overlap: one look at a table's entry per wavefront where all keys of a stage
// exist, instead of one per lane, took the prompts' call from 433 to 419 us, the reference kept as it is used to 411 to 416.  Four wavefronts of 64 rows read half as much from LDS, but one
// wavefront per SIMD has nothing to run beside its own vector instructions: 5500 cycles.
//
// The scores of the 32 keys after are multiplied while those of these are turned into probabilities, and
// the rest of the softmax is kept off the vector unit:
//  - the sum l is a product too, P with a row of ones (and so the sum of the rounded probabilities);
//  - there is no maximum in the common case.  The reference m of a row is set so that the largest probability is 2^-REF; a
//    later score may pass it, and only if a probability is then too large for the type's comfort (att_large) are
//    the maximum, the rescaling of O and l and the probabilities formed (again, from the keys, which are still in LDS).
//    A probability's precision is relative while it is a normal number: bf16 takes REF = 16 and lets a probability grow to 2, and
//    has normal numbers down to 2^-126; fp16, whose smallest is 2^-14 (2^-25 and less is nothing), takes -12 and lets one grow until
//    it is infinite, so that what lies less than 2^26 below a new maximum keeps all its bits.
template <int DP> struct AttTile {
  static constexpr int STAGE = DP == 256 ? 32 : 64;
  static constexpr int THREADS = 512, RING = 4, IDS = 1024, LDS = RING * 2 * STAGE * DP * 2 + IDS * 4;
};
__device__ const u32x4_t att_zeros = {0u, 0u, 0u, 0u};

// Whether a probability needs a new reference: a running value over packed pairs, and its test.  bf16: one of 2 or more
// has a bit of its own.  fp16: one that is infinite (above 65504), found behind the pairs' maximum.  Infinity and NaN count in both.
template <int DT> __device__ __forceinline__ uint32_t att_larger(uint32_t any, uint32_t lo, uint32_t hi) {
  if constexpr (DT == DT_F16) {
    typedef unsigned short pair_t __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_elementwise_max(__builtin_bit_cast(pair_t, lo), __builtin_bit_cast(pair_t, hi)), __builtin_bit_cast(pair_t, any)));
  } else return any | lo | hi;
}
template <int DT> __device__ __forceinline__ bool att_large(uint32_t any) {
  if constexpr (DT == DT_F16) return ((any | (any + 0x04000400u)) & 0x80008000u) != 0;
  else return (any & 0x40004000u) != 0;
}

// 16 bytes per lane from memory into LDS, to `to` (the same in every lane) + 16 lane.  In asm (nothing but LDS is written; the
// waits are written out where they belong) because with the compiler's own such load in flight every wait for an
// operand from LDS becomes one for all of them.
__device__ __forceinline__ uint32_t lds_at(void *to) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_readfirstlane((uint32_t)(__attribute__((address_space(3))) unsigned char *)to);
#else
  (void)to; return 0;
#endif
}
__device__ __forceinline__ void load_to_lds(const void *from, void *to) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_at(to)), "v"(from) : "memory", "m0");
#else
  (void)from; (void)to;
#endif
}
// the same with an address that is the wavefront's (see settled) and a lane's offset
__device__ __forceinline__ void load_to_lds(const void *from, uint32_t offset, void *to) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_at(to)), "v"(offset), "s"(from) : "memory", "m0");
#else
  (void)from; (void)offset; (void)to;
#endif
}
// Five wait states, after which a lane's value that was read into scalar registers right before may be a load's address: the
// compiler keeps them for its own loads, and does not see into the asm.
__device__ __forceinline__ void settled(const char *&a, const char *&b) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_nop 4" : "+s"(a), "+s"(b));
#else
  (void)a; (void)b;
#endif
}
// Lanes 4 r + c of sixteen address 8 bytes (columns 4 c .. 4 c + 3) of row r < 4; lane j gets column j of the four rows.
__device__ __forceinline__ uint2 read_transposed(const unsigned char *p) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef short s16x4_t __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)p));
#else
  (void)p;
  return make_uint2(0u, 0u);
#endif
}

template <int DT, int DP, bool FULL, bool POW2, int RT>
__global__ __launch_bounds__(512, 2) void tree_attention_tile_kernel(const AttParams P) {
  using C = AttTile<DP>;
  constexpr int ROWS = 128 * RT, STAGE = C::STAGE, THREADS = C::THREADS;
  constexpr int KS = DP / 32, NF = DP / 16;      // k steps of the first product, feature blocks of the second
  constexpr int CH = DP / 8, ROWB = DP * 2;      // 16-byte pieces and bytes of a row in LDS
  constexpr int SW = (CH < 16 ? CH : 16) - 1;
  constexpr int WROWS = STAGE / 8;               // rows of K (of V) that a wavefront loads of a stage
  constexpr int RPI = 64 / CH, NL = WROWS / RPI; // rows of one load instruction, load instructions
  constexpr int HALVES = STAGE / 32;
  constexpr int BUF = STAGE * ROWB;              // bytes of K (of V) of a stage
  constexpr float REF = DT == DT_F16 ? -12.0f : 16.0f, NONE = 3.402823466e38f, FAR = 16777216.0f;
  constexpr uint32_t ONES = DT == DT_F16 ? 0x3c003c00u : 0x3f803f80u;
  static_assert(NL * RPI == WROWS, "whole load instructions");
  extern __shared__ __attribute__((aligned(16))) unsigned char att_smem[];       // [RING][K, V][STAGE][ROWB], [IDS]
  int *ids = reinterpret_cast<int *>(att_smem + C::RING * 2 * BUF);              // the sequence's blocks from page0 on
  __shared__ long long scan[THREADS / 64];
  __shared__ long long found[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, quarter = lane >> 4;
  const int D = FULL ? DP : P.head_dim;
  const int share = run_tile_of(blockIdx.x, P.n_shares);
  AttRun<ROWS, STAGE, THREADS> run;
  if (tid == 0) P.joins[share] = make_int4(-1, 0, 0, 0);
  if (!run.begin(P, share, scan, found)) return;                   // (the same in every thread)

  // byte offset of this lane's operand of K in 16 rows, for the first k step; for step ks its bits of 64 ks are the other way
  const int kbase = col * ROWB + ((quarter ^ (col & SW)) * 16);
  const int vrow = 4 * quarter + (col >> 2);     // row of 16 that this lane addresses in a transposing read of V
  const int vswz = (((col & 3) >> 1) ^ (vrow & SW)) * 16, vbase = vrow * ROWB + (col & 1) * 8;
  const u32x4_t ones = {ONES, ONES, ONES, ONES};

  do {
    const AttSeq seq = run.seq;
    const int s = run.s, h = run.h, tile = run.tile, u0 = run.from(), u1 = run.to();
    const int n_rows = seq.n * P.group - tile * ROWS < ROWS ? seq.n * P.group - tile * ROWS : ROWS;   // of this tile
    const bool mine = wave * RT * 16 < n_rows;   // this wavefront has rows
    u32x4_t qf[RT][KS];
    int token[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int r = (wave * RT + rt) * 16 + col, gr = tile * ROWS + r;
      const int j = gr / P.group, hh = gr - j * P.group;
      token[rt] = j;
      const uint16_t *qp = P.q + (long long)(seq.row0 + j) * P.ldq + (long long)(h * P.group + hh) * D + quarter * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qf[rt][ks] = u32x4_t{0u, 0u, 0u, 0u};
        if (r < n_rows && (FULL || ks * 32 + quarter * 8 < D)) qf[rt][ks] = *reinterpret_cast<const u32x4_t *>(qp + ks * 32);
      }
    }
    f32x4_t o[RT][NF], l[RT];
    float ref[RT];                               // -m; NONE, fp32's largest number, where a row has seen no key yet: any score but minus infinity then makes an infinity
    bool far_off = false;                        // some row's reference is FAR or more in size (see below)
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      ref[rt] = NONE; l[rt] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int f = 0; f < NF; ++f) o[rt][f] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const int keys_end = att_tile_keys<ROWS>(P, seq, tile);                   // at least 1
    const int keys_all = P.mask ? seq.ctx : seq.ctx + tile * ROWS / P.group + 1;
    const int *table = P.table + (long long)s * P.table_pitch;
    const char *kh = reinterpret_cast<const char *>(P.k + (long long)h * D), *vh = reinterpret_cast<const char *>(P.v + (long long)h * D);

    // The blocks of the keys to be loaded are read from the table ahead, IDS at a time, into LDS: a wait for a list in
    // memory would be one for the rows in flight too.  Every wavefront calls this, between barriers.  clean: all blocks
    // so far exist.
    int page0 = 0;
    bool clean = true;
    auto fetch_ids = [&](int k0) {
      page0 = k0 / P.block_tokens;
      const int last = (keys_end - 1) / P.block_tokens;
      bool bad = false;
      for (int x = tid; x < C::IDS; x += THREADS) {
        const int id = table[page0 + x < last ? page0 + x : last];
        bad |= id < 0 || id >= P.n_pool_blocks;
        ids[x] = id;
      }
      if constexpr (FULL && POW2) {
        if (__syncthreads_or(bad)) clean = false;
      } else {
        __syncthreads();
      }
    };
    // The wavefront's rows of K and of V of the stage of keys from k0 on into place b of the ring: 2 NL load instructions,
    // whatever keys there are, so that the waits below can count them.  Keys that do not exist are rows of zeros.
    // Returns the keys that exist.
    auto issue = [&](int b, int k0) -> uint64_t {
      unsigned char *kb = att_smem + b * 2 * BUF + wave * WROWS * ROWB, *vb = kb + BUF;
      int ln = lane;                             // (the few instructions anew each time: kept through the loop they cost registers)
      // piece at place ln % CH of row ln / CH + RPI i of the wavefront's, which is row (WROWS wave + that) of the stage
      auto row_of = [&](int i) { return ln / CH + RPI * i; };
      auto piece_of = [&](int i) { return (uint32_t)((ln % CH) ^ ((WROWS * wave + row_of(i)) & SW)); };
      if (FULL && POW2 && clean && k0 + STAGE <= keys_end) {
        // nearly always: the wavefront's rows lie in one block, and every key of the stage exists
        asm volatile("" : "+v"(ln));
        const int kw = k0 + WROWS * wave;
        const int id = __builtin_amdgcn_readfirstlane(ids[(kw >> P.block_shift) - page0]);
        const uint64_t row0 = (uint32_t)((id << P.block_shift) + (kw & (P.block_tokens - 1)));
        const char *kr = kh + row0 * P.ldk, *vr = vh + row0 * P.ldv;
        settled(kr, vr);
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          load_to_lds(kr, row_of(i) * P.ldk + piece_of(i) * 16, kb + i * 1024);
          load_to_lds(vr, row_of(i) * P.ldv + piece_of(i) * 16, vb + i * 1024);
        }
        return STAGE == 64 ? ~0ull : 0xffffffffull;
      }
      const int kk = k0 + (lane & (STAGE - 1)), ke = kk < keys_end ? kk : keys_end - 1;
      const int page = POW2 ? ke >> P.block_shift : ke / P.block_tokens, off = POW2 ? ke & (P.block_tokens - 1) : ke - page * P.block_tokens;
      const int id = ids[page > page0 ? page - page0 : 0];         // (behind the last stage nothing is read ahead)
      const bool ok = kk < keys_end && id >= 0 && id < P.n_pool_blocks;
      uint64_t live = __ballot(ok);
      if constexpr (STAGE == 32) live &= 0xffffffffull;
      const int slot = ok ? (POW2 ? (id << P.block_shift) + off : id * P.block_tokens + off) : 0;
      const uint32_t here = (uint32_t)(live >> (WROWS * wave)) & ((1u << WROWS) - 1u);
      const uint64_t row0 = (uint32_t)__builtin_amdgcn_readlane(slot, WROWS * wave);
      asm volatile("" : "+v"(ln));
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int r = row_of(i);
        const uint32_t piece = piece_of(i);
        const char *kr, *vr;
        if constexpr (POW2) {
          kr = kh + row0 * P.ldk + (r * P.ldk + piece * 16);
          vr = vh + row0 * P.ldv + (r * P.ldv + piece * 16);
        } else {
          const uint64_t row = (uint32_t)__shfl(slot, WROWS * wave + r, 64);
          kr = kh + row * P.ldk + piece * 16;
          vr = vh + row * P.ldv + piece * 16;
        }
        const bool there = ((here >> r) & 1u) && (FULL || (int)piece * 8 < D);
        load_to_lds(there ? kr : reinterpret_cast<const char *>(&att_zeros), kb + i * 1024);
        load_to_lds(there ? vr : reinterpret_cast<const char *>(&att_zeros), vb + i * 1024);
      }
      return live;
    };
    // operands of the keys 16 u .. 16 u + 15 of the stage at kb (kx: kbase), and their scores
    auto read_k = [&](const unsigned char *kb, int kx, u32x4_t (&kf)[KS], int u) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) kf[ks] = *reinterpret_cast<const u32x4_t *>(kb + u * 16 * ROWB + (kx ^ (ks * 64)));
    };
    auto scores = [&](const u32x4_t (&kf)[KS], f32x4_t (&x)[RT][2], int u) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) x[rt][u] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) x[rt][u] = mfma16<DT>(kf[ks], qf[rt][ks], x[rt][u]);
    };

    const int k_first = u0 * STAGE, k_last = u1 * STAGE < keys_end ? u1 * STAGE : keys_end;
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();                // (the tile before has been read, and its last loads have landed)
    asm volatile("" ::: "memory");
    fetch_ids(k_first);
    uint64_t live0 = issue(0, k_first), live1 = issue(1, k_first + STAGE), live2 = issue(2, k_first + 2 * STAGE);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(4 * NL) : "memory");
    __builtin_amdgcn_s_barrier();                // stage 0 has landed
    asm volatile("" ::: "memory");
    f32x4_t sc[RT][2];                           // scores of the next 32 keys
    if (mine) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        u32x4_t kf[KS];
        read_k(att_smem, kbase, kf, u);
        scores(kf, sc, u);
      }
    }
    int b = 0;
    for (int k0 = k_first; k0 < k_last; k0 += STAGE, b = (b + 1) & 3) {
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * NL) : "memory");      // my rows of the next stage have landed
      __builtin_amdgcn_s_barrier();                                                  // everybody's have; the stage before has been read
      asm volatile("" ::: "memory");
      // (ids of the stage's last key; three stages lie within IDS from the first)
      const int ahead = k0 + 4 * STAGE - 1 < keys_end ? k0 + 4 * STAGE - 1 : keys_end - 1;
      if ((POW2 ? ahead >> P.block_shift : ahead / P.block_tokens) >= page0 + C::IDS) fetch_ids(k0 + 3 * STAGE);
      const uint64_t live3 = issue((b + 3) & 3, k0 + 3 * STAGE);
      const unsigned char *kb = att_smem + b * 2 * BUF, *vb = kb + BUF, *kb_next = att_smem + ((b + 1) & 3) * 2 * BUF;
      const uint64_t now = live0;
      live0 = live1; live1 = live2; live2 = live3;
      const bool masked = now != (STAGE == 64 ? ~0ull : 0xffffffffull) || k0 + STAGE > keys_all;
      if (!mine) continue;
      bool odd_v = false;
      if (masked) {                              // is there a value that is infinite or NaN?
#pragma unroll 1
        for (int x = 0; x < BUF / 1024; ++x) {
          const u32x4_t v = *reinterpret_cast<const u32x4_t *>(vb + x * 1024 + lane * 16);
#pragma unroll
          for (int w = 0; w < 4; ++w) odd_v |= not_finite<DT>(v[w]);
        }
        odd_v = __any(odd_v);
      }
#pragma unroll
      for (int c = 0; c < HALVES; ++c) {         // 32 keys
        int kx = kbase, vx = vbase, vz = vswz, q4 = 4 * quarter;
        asm volatile("" : "+v"(kx), "+v"(vx), "+v"(vz), "+v"(q4));      // (what is made of these is not kept through the loop)
        const unsigned char *kn = c + 1 < HALVES ? kb + (c + 1) * 32 * ROWB : kb_next;      // the 32 keys after these
        // Operands are read from LDS one group of matrix instructions ahead, which the barriers for the scheduler keep that
        // way: left to itself it reads each right before its use.
        u32x4_t kf[2][KS];
        read_k(kn, kx, kf[0], 0);
        uint32_t sees[RT];
        auto hide = [&](f32x4_t (&x)[RT][2]) {
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (!((sees[rt] >> (16 * u + q4 + i)) & 1u)) x[rt][u][i] = -__builtin_inff();
        };
        if (masked) {
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            int t = token[rt];
            asm volatile("" : "+v"(t));
            sees[rt] = att_window(P, seq, k0 + 32 * c, t, (wave * RT + rt) * 16 + col < n_rows) & (uint32_t)(now >> (32 * c));
          }
          hide(sc);
        }
        // ---- probabilities of these keys (rounded to the type: off by at most half a step, which is what the
        // output's own rounding is off by), beside the scores of the next
        u32x4_t pf[RT];
        uint32_t any = 0;
        auto probabilities = [&](const f32x4_t (&x)[RT][2], int u) {
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            float p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = att_exp2(fmaf(x[rt][u][i], P.scale2, ref[rt]));
            const uint32_t lo = pack2<DT>(p[0], p[1]), hi = pack2<DT>(p[2], p[3]);
            pf[rt][2 * u] = lo; pf[rt][2 * u + 1] = hi;
            any = att_larger<DT>(any, lo, hi);
          }
        };
        probabilities(sc, 0);
        read_k(kn, kx, kf[1], 1);
        __builtin_amdgcn_sched_barrier(0);
        scores(kf[0], sc, 0);
        probabilities(sc, 1);
        __builtin_amdgcn_sched_barrier(0);
        scores(kf[1], sc, 1);
        if (__any(att_large<DT>(any)) || far_off) {
          f32x4_t x[RT][2];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            u32x4_t kr[KS];
            read_k(kb, kx, kr, 2 * c + u);
            scores(kr, x, u);
          }
          if (masked) hide(x);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            float top = x[rt][0][0];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
              for (int i = 0; i < 4; ++i) top = fmaxf(top, x[rt][u][i]);
            top = quarters_max(top) * P.scale2;
            // The fused product above has more bits than the rounded one that the reference is made of: beside a reference of 2^24 (FAR)
            // the difference is a factor of up to 2, beside one of 2^31 an infinity or nothing.  From FAR on the wavefront rounds the
            // products, takes the maximum of every 32 keys, and a row's largest probability is 1.
            const bool seen = top != -__builtin_inff(), far = seen && fabsf(top) >= FAR;
            far_off |= __any(far) != 0;
            const float ref_new = !seen ? ref[rt] : fminf(ref[rt], far ? -top : -(top + REF));
            const float a = att_exp2(ref_new - ref[rt]);       // (0 from NONE on)
            ref[rt] = ref_new;
#pragma unroll
            for (int i = 0; i < 4; ++i) l[rt][i] *= a;
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[rt][f][i] *= a;
          }
          if (far_off) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                float p[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  float t = x[rt][u][i] * P.scale2;
                  asm volatile("" : "+v"(t));    // (not fused with the sum)
                  p[i] = att_exp2(t + ref[rt]);
                }
                pf[rt][2 * u] = pack2<DT>(p[0], p[1]); pf[rt][2 * u + 1] = pack2<DT>(p[2], p[3]);
              }
          } else {
#pragma unroll
            for (int u = 0; u < 2; ++u) probabilities(x, u);
          }
        }
        if (!odd_v) {
          uint2 va[2][2];
          auto read_v = [&](uint2 (&v)[2], int f) {
            const unsigned char *vp = vb + 32 * c * ROWB + vx + ((f * 32) ^ vz);
            v[0] = read_transposed(vp); v[1] = read_transposed(vp + 16 * ROWB);
          };
          read_v(va[0], 0);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) l[rt] = mfma16<DT>(ones, pf[rt], l[rt]);
#pragma unroll
          for (int f = 0; f < NF; ++f) {
            if (f + 1 < NF) read_v(va[(f + 1) & 1], f + 1);
            __builtin_amdgcn_sched_barrier(0);
            const uint2 (&v)[2] = va[f & 1];
            const u32x4_t vf = {v[0].x, v[0].y, v[1].x, v[1].y};
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) o[rt][f] = mfma16<DT>(vf, pf[rt], o[rt][f]);
          }
        } else {
          // 0 x infinity is no number: with such a value among the keys, every row adds up the keys that it sees, one by one
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) l[rt] = mfma16<DT>(ones, pf[rt], l[rt]);
#pragma unroll 1
          for (int kk = 0; kk < 32; ++kk) {
            const int x0 = 4 * (kk >> 4) + (kk & 3);         // which of the lane's probabilities
            float pk[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
              uint32_t w = 0;
#pragma unroll
              for (int x = 0; x < 4; ++x) w |= (x0 >> 1) == x ? pf[rt][x] : 0u;
              pk[rt] = __shfl(x0 & 1 ? hi_f32<DT>(w) : lo_f32<DT>(w), ((kk >> 2) & 3) * 16 + col, 64);
            }
#pragma unroll
            for (int f = 0; f < NF; ++f) {
              int qq = quarter;
              asm volatile("" : "+v"(qq));       // (an address of its own each time, not 2 NF running ones)
              const uint2 v = *reinterpret_cast<const uint2 *>(vb + (32 * c + kk) * ROWB + (((2 * f + (qq >> 1)) ^ (kk & SW)) * 16) + (qq & 1) * 8);
              const float x[4] = {lo_f32<DT>(v.x), hi_f32<DT>(v.x), lo_f32<DT>(v.y), hi_f32<DT>(v.y)};
#pragma unroll
              for (int rt = 0; rt < RT; ++rt)
                if ((sees[rt] >> kk) & 1u) {
#pragma unroll
                  for (int i = 0; i < 4; ++i) o[rt][f][i] += pk[rt] * x[i];
                }
            }
          }
        }
      }
    }

    // ---- out: to the rows, where this workgroup had all their keys, else to the workspace
    const bool whole = u0 == 0 && u1 == run.per_tile;
    const long long which = 2LL * share + (u0 == 0 ? 1 : 0);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int r = (wave * RT + rt) * 16 + col;
      if (r >= n_rows) continue;
      const float ll = l[rt][0];
      if (whole) {
        const int gr = tile * ROWS + r, hh = gr - token[rt] * P.group;
        uint16_t *op = P.out + (long long)(seq.row0 + token[rt]) * P.ldo + (long long)(h * P.group + hh) * D + 4 * quarter;
        const float inv = ll > 0.0f || ll != ll ? 1.0f / ll : 0.0f;               // (no key seen: zeros)
#pragma unroll
        for (int f = 0; f < NF; ++f)
          if (FULL || 16 * f + 4 * quarter < D)
            *reinterpret_cast<uint2 *>(op + 16 * f) = make_uint2(pack2<DT>(o[rt][f][0] * inv, o[rt][f][1] * inv), pack2<DT>(o[rt][f][2] * inv, o[rt][f][3] * inv));
      } else {
        float *pp = P.part + (which * ROWS + r) * DP + 4 * quarter;
#pragma unroll
        for (int f = 0; f < NF; ++f) *reinterpret_cast<f32x4_t *>(pp + 16 * f) = o[rt][f];
        if (quarter == 0) P.part_ml[which * ROWS + r] = make_float2(ref[rt] == NONE ? -__builtin_inff() : -ref[rt], ll);
      }
    }
    if (!whole && u0 == 0 && tid == 0) P.joins[share] = make_int4(s, h, tile, run.sharers());
  } while (run.next(P));
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // (rows loaded ahead and not used: their place in LDS is this workgroup's until they land)
}

// Joins the partial results of the tiles of rows whose keys several workgroups had: workgroup b takes the tile
// that begins in share b, whose other parts are the first of the shares after it, sixteen rows of it per workgroup.  Threads: (group of parts) x
// (row, 4 features); the groups' sums are joined in LDS in a fixed order.  4 us for tiles of 16 rows, a launch's and a
// dependent chain's (6 with one load after the other); 18 us for the 256-row tiles of 16 sequences, whose parts are some 60 MB written and
// read (one workgroup per tile took 45).
template <int ROWS> constexpr int JOIN_THREADS = ROWS == 16 ? 1024 : 256;
template <int DT, int DP, int ROWS>
__global__ __launch_bounds__(JOIN_THREADS<ROWS>) void tree_attention_join_kernel(const AttParams P) {
  const int share = blockIdx.x;
  const int4 job = P.joins[share];
  if (job.x < 0) return;
  constexpr int THREADS = JOIN_THREADS<ROWS>, QUADS = DP / 4, ITEMS = 16 * QUADS;
  constexpr int SETS = ITEMS < THREADS ? THREADS / ITEMS : 1, AHEAD = ROWS == 16 ? 4 : 2;      // (large tiles have few parts)
  __shared__ __attribute__((aligned(16))) float sum_o[SETS > 1 ? SETS * 16 * DP : 4];
  __shared__ float sum_l[SETS > 1 ? SETS * 16 : 1];
  const AttSeq seq = att_seq(P, job.x);
  const int h = job.y, tile = job.z, parts = job.w, tid = threadIdx.x;
  const int n_rows = seq.n * P.group - tile * ROWS < ROWS ? seq.n * P.group - tile * ROWS : ROWS;
  auto part_at = [&](int i, int r) -> long long { return ((long long)(2 * (share + i)) + (i == 0 ? 1 : 0)) * ROWS + r; };
  const int r0 = blockIdx.y * 16;
  if (r0 >= n_rows) return;
  for (int x = tid; x < SETS * ITEMS; x += THREADS) {
    const int set = x / ITEMS, item = x - set * ITEMS, rr = item / QUADS, d = (item - rr * QUADS) * 4, r = r0 + rr;
    float mm = -__builtin_inff(), ll = 0.0f;
    f32x4_t y = {0.0f, 0.0f, 0.0f, 0.0f};
    if (r < n_rows) {
      // (AHEAD loads side by side: the last part stands in for those behind it, and is not added)
      for (int i0 = 0; i0 < parts; i0 += 2 * AHEAD) {
        float x[2 * AHEAD];
#pragma unroll
        for (int i = 0; i < 2 * AHEAD; ++i) x[i] = P.part_ml[part_at(i0 + i < parts ? i0 + i : parts - 1, r)].x;
#pragma unroll
        for (int i = 0; i < 2 * AHEAD; ++i) mm = fmaxf(mm, x[i]);
      }
      for (int i0 = set; i0 < parts; i0 += SETS * AHEAD) {
        float2 ml[AHEAD];
        f32x4_t z[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
          const long long at = part_at(i0 + SETS * i < parts ? i0 + SETS * i : parts - 1, r);
          ml[i] = P.part_ml[at];
          z[i] = *reinterpret_cast<const f32x4_t *>(P.part + at * DP + d);
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
          if (i0 + SETS * i >= parts) continue;
          const float a = ml[i].x == -__builtin_inff() ? 1.0f : att_exp2(ml[i].x - mm);
          ll += a * ml[i].y;
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] += a * z[i][e];
        }
      }
    }
    if constexpr (SETS > 1) {
      *reinterpret_cast<f32x4_t *>(sum_o + (set * 16 + rr) * DP + d) = y;
      if (d == 0) sum_l[set * 16 + rr] = ll;
      __syncthreads();                                          // (one pass of the loop: SETS * ITEMS == THREADS)
      if (set == 0) {
        ll = 0.0f; y = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < SETS; ++w) {
          ll += sum_l[w * 16 + rr];
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] += sum_o[(w * 16 + rr) * DP + d + e];
        }
      }
      __syncthreads();
    }
    if (set == 0 && r < n_rows && d < P.head_dim) {
      const int gr = tile * ROWS + r, j = gr / P.group, hh = gr - j * P.group;
      const float inv = ll > 0.0f || ll != ll ? 1.0f / ll : 0.0f;
      *reinterpret_cast<uint2 *>(P.out + (long long)(seq.row0 + j) * P.ldo + (long long)(h * P.group + hh) * P.head_dim + d) =
          make_uint2(pack2<DT>(y[0] * inv, y[1] * inv), pack2<DT>(y[2] * inv, y[3] * inv));
    }
  }
}

}  // namespace deinfer
