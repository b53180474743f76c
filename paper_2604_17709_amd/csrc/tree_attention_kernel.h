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
  long long ldq, ldk, ldv, ldo, table_pitch, n_pool_blocks, most_keys;     // most_keys: tokens that a row of the table can hold
  int T, n_seqs, n_kv, group, head_dim, block_tokens, block_shift, mask_words;
  float scale2;                                  // scale log2(e): the exponentials are powers of two
  int n_shares;
  float *part;                                   // [2 n_shares][rows][DP] partial outputs
  float2 *part_ml;                               // [2 n_shares][rows] their maxima and sums
  int4 *joins;                                   // [n_shares] tile of rows whose first share this is and that others share (sequence, head, tile, shares)
};

struct AttSeq { int row0, n, ctx; long long keys; };             // first row, rows, cached tokens, keys in all
__device__ __forceinline__ AttSeq att_seq(const AttParams &P, int s) {
  AttSeq q;
  int r0 = P.row_start[s], r1 = P.row_start[s + 1];
  r0 = r0 < 0 ? 0 : r0; r1 = r1 > P.T ? P.T : r1;
  q.row0 = r0; q.n = r1 > r0 ? r1 - r0 : 0;
  const int c = P.cached[s];
  q.ctx = c < 0 ? 0 : c;
  const long long keys = (long long)q.ctx + q.n;
  q.keys = keys < P.most_keys ? keys : P.most_keys;
  return q;
}
template <int ROWS, int UNIT> struct AttTiles {                   // units of one sequence
  long long units; int tiles, per_tile;
  __device__ __forceinline__ AttTiles(const AttSeq &q, int group, int n_kv) {
    tiles = (int)(((long long)q.n * group + ROWS - 1) / ROWS);
    per_tile = (int)((q.keys + UNIT - 1) / UNIT);
    per_tile = per_tile < 1 ? 1 : per_tile;                       // (rows without any key are written too)
    units = (long long)n_kv * tiles * per_tile;
  }
};

// a value that is the same in every lane, in scalar registers
__device__ __forceinline__ long long uniform(long long x) {
  return ((long long)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x);
}
__device__ __forceinline__ float att_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
// the larger (the sum) of the four quarters of the wave, in every lane
__device__ __forceinline__ float quarters_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16, 64));
  return fmaxf(x, __shfl_xor(x, 32, 64));
}
__device__ __forceinline__ float quarters_sum(float x) {
  x += __shfl_xor(x, 16, 64);
  return x + __shfl_xor(x, 32, 64);
}

// 16-bit elements of a word that are infinite or NaN
template <int DT> __device__ __forceinline__ bool not_finite(uint32_t w) {
  constexpr uint32_t E = DT == DT_F16 ? 0x7c00u : 0x7f80u;
  return (w & E) == E || (w & (E << 16)) == (E << 16);
}

// DP: head dimension up to 64, 128 or 256; FULL: it is DP; POW2: blocks of a power of two of at least 16
// tokens (16 neighbouring keys are rows of one block: their address is one scalar and a lane's constant);
// WR x WK wavefronts, WR row groups of RT tiles of 16 rows, each over WK interleaved shares of the keys.
template <int DT, int DP, bool FULL, bool POW2, int WR, int WK, int RT>
__global__ __launch_bounds__(ATT_THREADS) void tree_attention_kernel(const AttParams P) {
  static_assert(WR * WK * 64 == ATT_THREADS, "four wavefronts");
  constexpr int ROWS = 16 * WR * RT, UNIT = ATT_KEYS * WK;
  constexpr int KS = DP / 32;                    // k steps of the first product
  constexpr int VE = DP == 64 ? 4 : 8;           // neighbouring features of V per lane and piece
  constexpr int NC = DP / (16 * VE);             // pieces
  constexpr int NF = NC * VE;                    // 16-feature blocks of the output
  constexpr int VW = VE / 2;                     // words of a piece
  constexpr int OP = DP + 4;                     // row pitch of the merge buffer in LDS
  __shared__ __attribute__((aligned(16))) float merge_o[WK > 1 ? WK * 16 * OP : 4];
  __shared__ float merge_ml[WK > 1 ? 2 * WK * 16 : 2];
  __shared__ long long scan[ATT_THREADS / 64];
  __shared__ long long found[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = wave / WK, wk = wave % WK;
  const int col = lane & 15, quarter = lane >> 4;
  const int D = FULL ? DP : P.head_dim;
  const int share = run_tile_of(blockIdx.x, P.n_shares);

  // ---- my run of units
  auto units_of = [&](int s) -> long long {
    if (s >= P.n_seqs) return 0;
    return AttTiles<ROWS, UNIT>(att_seq(P, s), P.group, P.n_kv).units;
  };
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
    for (int w = 0; w < ATT_THREADS / 64; ++w) { if (w < wave) before += scan[w]; all += scan[w]; }
    *total = all;
    return u + before;
  };
  long long total = 0;
  for (int s0 = 0; s0 < P.n_seqs; s0 += ATT_THREADS) {
    long long t;
    scan_units(units_of(s0 + tid), &t);
    total += t;
  }
  total = uniform(total);
  const long long per_share = (total + P.n_shares - 1) / P.n_shares;
  long long cur = per_share * share;
  const long long end = cur + per_share < total ? cur + per_share : total;
  if (tid == 0) P.joins[share] = make_int4(-1, 0, 0, 0);
  if (cur >= end) return;                                          // (the same in every thread)
  {
    long long base = 0;
    for (int s0 = 0; s0 < P.n_seqs; s0 += ATT_THREADS) {
      long long t;
      const long long u = units_of(s0 + tid), e = base + scan_units(u, &t);
      if (u > 0 && e - u <= cur && cur < e) { found[0] = s0 + tid; found[1] = e - u; }
      base += t;
      if (base > cur) break;
    }
    __syncthreads();
  }
  int s = __builtin_amdgcn_readfirstlane((int)found[0]);
  long long seq_base = uniform(found[1]);

  while (cur < end) {
    const AttSeq seq = att_seq(P, s);
    const AttTiles<ROWS, UNIT> ti(seq, P.group, P.n_kv);
    if (cur >= seq_base + ti.units) { seq_base += ti.units; ++s; continue; }
    const long long in_seq = cur - seq_base;
    const int h = (int)(in_seq / ((long long)ti.tiles * ti.per_tile));
    const long long in_head = in_seq - (long long)h * ti.tiles * ti.per_tile;
    const int tile = (int)(in_head / ti.per_tile), u0 = (int)(in_head - (long long)tile * ti.per_tile);
    const int u1 = end - cur < ti.per_tile - u0 ? u0 + (int)(end - cur) : ti.per_tile;

    // ---- the rows
    const int n_rows = seq.n * P.group - tile * ROWS < ROWS ? seq.n * P.group - tile * ROWS : ROWS;   // of this tile
    u32x4_t qf[RT][KS];
    int token[RT];                               // of this lane's row of every row tile
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int r = (wr * RT + rt) * 16 + col, gr = tile * ROWS + r;
      const int j = gr / P.group, hh = gr - j * P.group;
      token[rt] = j;
      const uint16_t *qp = P.q + (long long)(seq.row0 + j) * P.ldq + (long long)(h * P.group + hh) * D + quarter * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qf[rt][ks] = u32x4_t{0u, 0u, 0u, 0u};
        if (r < n_rows && (FULL || ks * 32 + quarter * 8 < D)) qf[rt][ks] = *reinterpret_cast<const u32x4_t *>(qp + ks * 32);
      }
    }
    f32x4_t o[RT][NF];
    float m[RT], l[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      m[rt] = -__builtin_inff(); l[rt] = 0.0f;
#pragma unroll
      for (int f = 0; f < NF; ++f) o[rt][f] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const int first_token = tile * ROWS / P.group, last_token = (tile * ROWS + n_rows - 1) / P.group;
    // keys that some row may see (a causal tile needs none behind its last token), and keys that every row sees
    long long keys_end = P.mask ? seq.keys : (long long)seq.ctx + last_token + 1;
    keys_end = keys_end < seq.keys ? keys_end : seq.keys;
    const long long keys_all = P.mask ? seq.ctx : (long long)seq.ctx + first_token + 1;

    const int *table = P.table + s * P.table_pitch;
    const int klane = col * (int)P.ldk + quarter * 8, vlane = quarter * 4 * (int)P.ldv + col * VE;
    for (long long k0 = (long long)u0 * UNIT + wk * ATT_KEYS; k0 < (long long)u1 * UNIT && k0 < keys_end; k0 += UNIT) {
      // ---- where the 32 keys are; `live`: those that exist
      uint32_t live = keys_end - k0 >= 32 ? 0xffffffffu : (1u << (int)(keys_end - k0)) - 1u;
      const uint16_t *kp[2], *vp[2];             // POW2: rows of the two halves' first keys
      long long slot = 0;                        // otherwise: row of the key k0 + lane % 32
      if constexpr (POW2) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const long long kk = k0 + 16 * u;
          int id = -1;
          if (kk < keys_end) id = table[kk >> P.block_shift];
          const bool ok = id >= 0 && id < P.n_pool_blocks;
          if (!ok) live &= ~(0xffffu << (16 * u));
          const long long row = ok ? ((long long)id << P.block_shift) + (kk & (P.block_tokens - 1)) : 0;
          kp[u] = P.k + row * P.ldk + (long long)h * D;
          vp[u] = P.v + row * P.ldv + (long long)h * D;
        }
      } else {
        const long long kk = k0 + (lane & 31);
        bool ok = false;
        if (kk < keys_end) {
          const long long page = kk / P.block_tokens;
          const int id = table[page];
          ok = id >= 0 && id < P.n_pool_blocks;
          if (ok) slot = (long long)id * P.block_tokens + (kk - page * P.block_tokens);
        }
        live &= (uint32_t)__ballot(ok);
      }
      u32x4_t kf[2][KS];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint16_t *kr;
        if constexpr (POW2) kr = kp[u] + klane;
        else kr = P.k + __shfl(slot, 16 * u + col, 64) * P.ldk + (long long)h * D + quarter * 8;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          kf[u][ks] = u32x4_t{0u, 0u, 0u, 0u};
          if (FULL || ks * 32 + quarter * 8 < D) kf[u][ks] = *reinterpret_cast<const u32x4_t *>(kr + ks * 32);
        }
      }
      uint32_t vw[NC][8][VW];                    // [piece][key 4 u + i of the lane][word]
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const uint16_t *vr;
        if constexpr (POW2) vr = vp[x / 4] + (vlane + (x % 4) * (int)P.ldv);
        else vr = P.v + __shfl(slot, 16 * (x / 4) + 4 * quarter + x % 4, 64) * P.ldv + (long long)h * D + col * VE;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
#pragma unroll
          for (int w = 0; w < VW; ++w) vw[c][x][w] = 0u;
          if (FULL || c * 16 * VE + col * VE < D) {
            if constexpr (VE == 8) {
              const u32x4_t t = *reinterpret_cast<const u32x4_t *>(vr + c * 128);
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
      uint32_t sees[RT];
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
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          uint32_t w = 0xffffffffu;
          if (!P.mask) {
            const long long n = (long long)seq.ctx + token[rt] + 1 - k0;
            w = n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << (int)n) - 1u;
          } else if (k0 + 32 > seq.ctx) {
            const long long e = k0 - seq.ctx;    // first key of the 32 as index among the step's tokens; > -32
            const uint32_t *mw = P.mask + (long long)(seq.row0 + token[rt]) * P.mask_words;
            const bool row = (wr * RT + rt) * 16 + col < n_rows;
            auto word = [&](long long i) -> uint32_t { return row && i < P.mask_words ? mw[i] : 0u; };
            if (e < 0) {
              w = (word(0) << (int)-e) | ((1u << (int)-e) - 1u);
            } else {
              const int sh = (int)(e & 31);
              w = word(e >> 5) >> sh;
              if (sh) w |= word((e >> 5) + 1) << (32 - sh);
            }
          }
          sees[rt] = w & live;
        }
      }
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        f32x4_t sc[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          sc[u] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) sc[u] = mfma16<DT>(kf[u][ks], qf[rt][ks], sc[u]);
        }
        float p[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) p[x] = sc[x / 4][x % 4] * P.scale2;
        if (masked) {
#pragma unroll
          for (int x = 0; x < 8; ++x)
            if (!((sees[rt] >> (16 * (x / 4) + 4 * quarter + x % 4)) & 1u)) p[x] = -__builtin_inff();
        }
        float top = p[0];
#pragma unroll
        for (int x = 1; x < 8; ++x) top = fmaxf(top, p[x]);
        top = quarters_max(top);
        if (__any(top > m[rt])) {
          const float m_new = fmaxf(m[rt], top);
          const float a = m[rt] == -__builtin_inff() ? 0.0f : att_exp2(m[rt] - m_new);
          m[rt] = m_new;
          l[rt] *= a;
#pragma unroll
          for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[rt][f][i] *= a;
        }
        const float base = m[rt] == -__builtin_inff() ? 0.0f : m[rt];     // (a row that has seen no key yet)
        float sum = 0.0f;
#pragma unroll
        for (int x = 0; x < 8; ++x) { p[x] = att_exp2(p[x] - base); sum += p[x]; }
        l[rt] += sum;
        // the probabilities, at most 1, as the 16-bit operand of the second product: each is off by at most half a
        // step of the type, which is what the output's own rounding is off by
        const u32x4_t pf = {pack2<DT>(p[0], p[1]), pack2<DT>(p[2], p[3]), pack2<DT>(p[4], p[5]), pack2<DT>(p[6], p[7])};
        if (!masked || !odd_v) {
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int e = 0; e < VE; ++e) {
              u32x4_t vf;
#pragma unroll
              for (int w = 0; w < 4; ++w)
                vf[w] = __builtin_amdgcn_perm(vw[c][2 * w + 1][e / 2], vw[c][2 * w][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
              o[rt][c * VE + e] = mfma16<DT>(vf, pf, o[rt][c * VE + e]);
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
            const bool see = (sees[rt] >> kk) & 1u;
            const uint16_t *vr;
            if constexpr (POW2) vr = (kk < 16 ? vp[0] : vp[1]) + (kk & 15) * P.ldv;
            else vr = P.v + __shfl(slot, kk, 64) * P.ldv + (long long)h * D;
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int d = (f / VE) * 16 * VE + (quarter * 4 + i) * VE + f % VE;
                if (see && (FULL || d < D)) o[rt][f][i] += pk * cvt_in<DT>(vr[d]);
              }
          }
        }
      }
    }

    // ---- out: to the rows, where this workgroup had all their keys, else to the workspace
    const bool whole = u0 == 0 && u1 == ti.per_tile;
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
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const float lsum = quarters_sum(l[rt]);
      if constexpr (WK == 1) {
        const int r = (wr * RT + rt) * 16 + col;
        if (r < n_rows) {
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int d = c * 16 * VE + (quarter * 4 + i) * VE;
              float x[VE];
#pragma unroll
              for (int e = 0; e < VE; ++e) x[e] = o[rt][c * VE + e][i];
              if (FULL || d < D) store_row(r, d, x, m[rt], lsum);
            }
        }
      } else {
        static_assert(WK == 1 || WR == 1, "the merge buffer is that of one row group");
        __syncthreads();                                            // (the buffer's last readers are done)
        if (quarter == 0) { merge_ml[(wk * 16 + col) * 2] = m[rt]; merge_ml[(wk * 16 + col) * 2 + 1] = lsum; }
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float *mp = merge_o + (wk * 16 + col) * OP + c * 16 * VE + (quarter * 4 + i) * VE;
#pragma unroll
            for (int e = 0; e < VE; e += 4)
              *reinterpret_cast<f32x4_t *>(mp + e) = f32x4_t{o[rt][c * VE + e][i], o[rt][c * VE + e + 1][i], o[rt][c * VE + e + 2][i], o[rt][c * VE + e + 3][i]};
          }
        __syncthreads();
        for (int x = tid; x < 16 * (DP / VE); x += ATT_THREADS) {
          const int rr = x / (DP / VE), d = (x - rr * (DP / VE)) * VE, r = rt * 16 + rr;
          if (r >= n_rows || (!FULL && d >= D)) continue;
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
          store_row(r, d, y, mm, ll);
        }
      }
    }
    if (!whole && u0 == 0 && tid == 0) {
      const long long first = cur, last = cur + ti.per_tile - 1;
      P.joins[share] = make_int4(s, h, tile, (int)(last / per_share - first / per_share + 1));
    }
    cur += u1 - u0;
  }
}

// Joins the partial results of the tiles of rows whose keys several workgroups had: workgroup b takes the tile
// that begins in share b, whose other parts are the first of the shares after it.  Threads: (group of parts) x
// (row, 4 features); the groups' sums are joined in LDS in a fixed order.
constexpr int JOIN_THREADS = 1024;
template <int DT, int DP, int ROWS>
__global__ __launch_bounds__(JOIN_THREADS) void tree_attention_join_kernel(const AttParams P) {
  const int share = blockIdx.x;
  const int4 job = P.joins[share];
  if (job.x < 0) return;
  constexpr int QUADS = DP / 4, ITEMS = 16 * QUADS;             // a pass takes 16 rows
  constexpr int SETS = ITEMS < JOIN_THREADS ? JOIN_THREADS / ITEMS : 1;
  __shared__ __attribute__((aligned(16))) float sum_o[SETS > 1 ? SETS * 16 * DP : 4];
  __shared__ float sum_l[SETS > 1 ? SETS * 16 : 1];
  const AttSeq seq = att_seq(P, job.x);
  const int h = job.y, tile = job.z, parts = job.w, tid = threadIdx.x;
  const int n_rows = seq.n * P.group - tile * ROWS < ROWS ? seq.n * P.group - tile * ROWS : ROWS;
  auto part_at = [&](int i, int r) -> long long { return ((long long)(2 * (share + i)) + (i == 0 ? 1 : 0)) * ROWS + r; };
  for (int r0 = 0; r0 < n_rows; r0 += 16) {
    for (int x = tid; x < SETS * ITEMS; x += JOIN_THREADS) {
      const int set = x / ITEMS, item = x - set * ITEMS, rr = item / QUADS, d = (item - rr * QUADS) * 4, r = r0 + rr;
      float mm = -__builtin_inff(), ll = 0.0f;
      f32x4_t y = {0.0f, 0.0f, 0.0f, 0.0f};
      if (r < n_rows) {
        for (int i = 0; i < parts; ++i) mm = fmaxf(mm, P.part_ml[part_at(i, r)].x);
        for (int i = set; i < parts; i += SETS) {
          const float2 ml = P.part_ml[part_at(i, r)];
          const float a = ml.x == -__builtin_inff() ? 1.0f : att_exp2(ml.x - mm);
          ll += a * ml.y;
          const f32x4_t z = *reinterpret_cast<const f32x4_t *>(P.part + part_at(i, r) * DP + d);
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] += a * z[e];
        }
      }
      if constexpr (SETS > 1) {
        *reinterpret_cast<f32x4_t *>(sum_o + (set * 16 + rr) * DP + d) = y;
        if (d == 0) sum_l[set * 16 + rr] = ll;
        __syncthreads();                                          // (one pass of the loop: SETS * ITEMS == JOIN_THREADS)
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
}

}  // namespace deinfer
