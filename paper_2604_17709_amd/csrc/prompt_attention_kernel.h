// Attention of packed prompts over packed keys and values: rows of q, k and v as the projections write them (or keys
// and values rebuilt from the low-rank cache), sequence after sequence, no pages.  Gaps between the keys of sequences, as the
// rebuilt cache has them, are sequences without rows, which have no tiles and no work.
//
// Token i of a sequence with n rows and K keys stands at p = K - n + i and sees the keys j with p - left <= j <= p + right,
//   o = sum_j exp(x_j - max x) v_j / sum_j exp(x_j - max x),   x_j = scale q . k_j,
// in one pass over the keys: a reference m, a running sum l and an unnormalised output O per row, all in fp32.
//
// A tile is `tile_tokens` tokens of a sequence with the query heads that share a key head: neighbouring heads use the same keys, so
// a tile of grouped heads has few tokens and little beyond its diagonal.  Its keys [F, E) are those that some row of it sees.
// Work is counted in keys of a tile, over all sequences, key heads and tiles, and START more per tile, what a tile costs beside
// its keys; every workgroup takes an equal run, found on the device from the lengths: the sums over a sequence's tiles are those of
// clamped arithmetic series, so the run is found by a scan over the sequences and a bisection.  A stage (UNIT keys) belongs to the
// workgroup whose run its last key falls into.  A tile whose stages several workgroups share leaves partial (O, m, l) in
// the workspace, at most two per workgroup, and a second launch joins them in order: results do not depend on timing.
#pragma once
#include "tree_attention_kernel.h"

namespace deinfer {

constexpr int PROMPT_FAR = 1 << 29;              // a window side without a bound

struct PromptParams {
  const uint16_t *q, *k, *v;
  uint16_t *out;
  const int *q_start, *k_start;
  long long ldq, ldo;
  uint32_t ldk, ldv;                             // in bytes
  int T, Tk, n_seqs, head_dim, group;
  int heads, head_tiles, tile_group, tile_tokens;      // key heads x parts of their query heads (head_tiles); query heads and tokens of a tile
  double per_token, per_workgroup;               // 1 / tile_tokens, 1 / n_shares
  int left, right;                               // at most PROMPT_FAR
  float scale2;                                  // scale log2(e): the exponentials are powers of two
  int n_shares;
  float *part;                                   // [2 n_shares][rows][columns] partial outputs
  float2 *part_ml;                               // [2 n_shares][rows] their references and sums
  int4 *joins;                                   // [n_shares] tile whose first share this is and that others share (sequence, head, tile, shares)
};

struct PromptSeq { int row0, n, key0, keys; };
__device__ __forceinline__ PromptSeq prompt_seq(const PromptParams &P, int s) {
  auto range = [&](const int *start, int most, int &from, int &count) {
    int a = start[s], b = start[s + 1];
    a = a < 0 ? 0 : a; b = b > most ? most : b;
    from = a; count = b > a ? b - a : 0;
  };
  PromptSeq q;
  range(P.q_start, P.T, q.row0, q.n);
  if (P.k_start) range(P.k_start, P.Tk, q.key0, q.keys);
  else range(P.q_start, P.Tk < P.T ? P.Tk : P.T, q.key0, q.keys);
  return q;
}
// keys of a tile: [first, first + count)
struct PromptKeys { int first, count; };
__device__ __forceinline__ PromptKeys prompt_keys(const PromptParams &P, const PromptSeq &q, int tile) {
  const int c0 = q.keys - q.n, t0 = tile * P.tile_tokens;
  const int t1 = q.n - t0 < P.tile_tokens ? q.n : t0 + P.tile_tokens;
  int a = c0 + t0 - P.left, b = c0 + t1 + P.right;
  a = a < 0 ? 0 : a > q.keys ? q.keys : a;
  b = b < 0 ? 0 : b > q.keys ? q.keys : b;
  return {a, b - a};
}
// sum over i < t of a + i step, each held within [0, most]; per_step: 1 / step (x + 1/2 is at least 1 / (2 step) steps from a whole number of them,
// and the product less than 2^-20 of that off)
__device__ __forceinline__ long long clamped_series(int a, int step, double per_step, int most, int t) {
  auto steps = [&](int x) { return x <= 0 ? 0 : (int)(((double)(x + step - 1) + 0.5) * per_step); };        // up to x, rounded up
  int z = steps(-a), f = steps(most - a);
  z = z > t ? t : z; f = f > t ? t : f;
  if (f <= z) return (long long)(t - f) * most;
  return (long long)(f - z) * a + ((long long)f * (f - 1) - (long long)z * (z - 1)) / 2 * step + (long long)(t - f) * most;
}
// work of a sequence's first t tiles of one head
template <int START> __device__ __forceinline__ long long prompt_work(const PromptParams &P, const PromptSeq &q, int t) {
  const int c0 = q.keys - q.n, step = P.tile_tokens;
  return (long long)t * START + clamped_series(c0 + step + P.right, step, P.per_token, q.keys, t) - clamped_series(c0 - P.left, step, P.per_token, q.keys, t);
}
__device__ __forceinline__ long long lane_value(long long x, int lane) {
  return (long long)(uint32_t)__builtin_amdgcn_readlane((int)x, lane) | (long long)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32;
}
// a / b where the quotient is an int: a division in 64-bit floating point is off by less than one then
__device__ __forceinline__ int small_quotient(long long a, long long b) {
  int q = (int)((double)a / (double)b);
  const long long r = a - q * b;
  return r < 0 ? q - 1 : r >= b ? q + 1 : q;
}
__device__ __forceinline__ int prompt_tiles(const PromptParams &P, const PromptSeq &q) { return (q.n + P.tile_tokens - 1) / P.tile_tokens; }

// The order of the work: sequence after sequence; in it chunks of heads; in a chunk pairs of tiles, the last with the first and
// so on inwards, whose work is about the same for every pair of a causal prompt; for a pair head after head; the later tile before
// the earlier.  A chunk has so many heads that a workgroup's run is one pair through all of them: at any time the workgroups of a
// chunk are at the same head, and read the same rows of K and V through one L2.  16 prompts of up to 2500 tokens with 32 heads of
// 128, fp16: 767 us causal and 1301 with all keys seen, against 796 and 1348 in the order of heads.
//
// A workgroup's run, tile after tile.  Everything is the same in all lanes.
template <int UNIT, int START, int THREADS> struct PromptRun {
  long long per_share, from_work, end, base;     // base: work ahead of the present tile's first key (behind its START)
  PromptSeq seq;
  int s, h, tile;
  int tiles, pair, chunk_heads, in_chunk;        // tiles of the sequence and head; present pair; heads of a chunk of the sequence; heads of this chunk from the present one on
  int chunk_first;                               // first head of the chunk
  PromptKeys keys;
  int k_from, k_to;                              // the workgroup's part of the present tile's keys, relative to keys.first

  // scan: THREADS / 64 values, found: 2 values of LDS.  False: nothing to do
  __device__ __forceinline__ bool begin(const PromptParams &P, int share, long long *scan, long long *found) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    auto before_lanes = [&](long long u) {       // inclusive sum over the wavefront's lanes
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const long long w = __shfl_up(u, o, 64);
        if (lane >= o) u += w;
      }
      return u;
    };
    auto shared_out = [&](long long total) {
      per_share = (long long)((double)total * P.per_workgroup * (1.0 + 0x1p-50)) + 1;  // (no less than the share, whatever the roundings)
      per_share = uniform(per_share < UNIT ? UNIT : per_share);      // (every share between a tile's first and last then has a stage's last key)
      from_work = per_share * share;
      end = from_work + per_share < total ? from_work + per_share : total;
      return from_work < end;
    };
    long long per_head;                          // work of the sequence for one head
    if (P.n_seqs <= 64) {
      // a sequence in every lane, and every wavefront for itself: nothing goes through LDS
      PromptSeq q = {0, 0, 0, 0};
      long long one = 0;
      if (lane < P.n_seqs) {
        q = prompt_seq(P, lane);
        one = prompt_work<START>(P, q, prompt_tiles(P, q));
      }
      const long long mine = P.heads * one, mine_end = before_lanes(mine);
      if (!shared_out(lane_value(mine_end, 63))) return false;
      const unsigned long long has = __ballot(mine > 0 && mine_end - mine <= from_work && from_work < mine_end);
      if (has == 0) return false;                // (lists of sequences that overlap so much that the sum of their work is beyond 64 bits)
      s = __builtin_ctzll(has);
      base = lane_value(mine_end - mine, s); per_head = lane_value(one, s);
      seq = {__builtin_amdgcn_readlane(q.row0, s), __builtin_amdgcn_readlane(q.n, s), __builtin_amdgcn_readlane(q.key0, s), __builtin_amdgcn_readlane(q.keys, s)};
    } else {
      auto work_of = [&](int x) -> long long {
        if (x >= P.n_seqs) return 0;
        const PromptSeq q = prompt_seq(P, x);
        return P.heads * prompt_work<START>(P, q, prompt_tiles(P, q));
      };
      auto scan_work = [&](long long u, long long *total) {          // inclusive sum over the threads
        u = before_lanes(u);
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
        mine = work_of(s0 + tid);
        mine_end = scan_work(mine, &t);
        total += t;
      }
      total = uniform(total);
      if (!shared_out(total)) return false;
      long long before = 0;
      if (tid == 0) found[0] = -1;
      __syncthreads();
      for (int s0 = 0; s0 < P.n_seqs; s0 += THREADS) {
        long long t = total;
        if (P.n_seqs > THREADS) {
          mine = work_of(s0 + tid);
          mine_end = scan_work(mine, &t);
        }
        const long long e = before + mine_end;
        if (mine > 0 && e - mine <= from_work && from_work < e) { found[0] = s0 + tid; found[1] = e - mine; }
        before += t;
        if (before > from_work) break;
      }
      __syncthreads();
      s = __builtin_amdgcn_readfirstlane((int)found[0]);
      base = uniform(found[1]);
      if (s < 0) return false;                   // (as above)
      seq = prompt_seq(P, s);
      per_head = uniform(prompt_work<START>(P, seq, prompt_tiles(P, seq)));
    }
    if (from_work < base || from_work - base >= P.heads * per_head) return false;        // (and again)
    enter(P, per_head);
    const int chunk = small_quotient(from_work - base, per_head * chunk_heads);
    chunk_first = chunk * chunk_heads;
    const int n = P.heads - chunk_first < chunk_heads ? P.heads - chunk_first : chunk_heads;
    base += (long long)chunk * chunk_heads * per_head;
    int lo = 0, most = (tiles + 1) / 2;          // the last pair that begins at or before from_work, among [lo, most): 64 of them at a time
    long long work;                              // in lane 0 and 1: of the pairs ahead of it, and with it
    for (;;) {
      const int rest = most - lo, step = (rest + 63) / 64, at = lo + lane * step;
      work = pairs_work(P, per_head, at);
      if (rest <= 1) break;
      const int c = __popcll(__ballot(at < most && base + n * work <= from_work)) - 1;
      lo += c > 0 ? c * step : 0;
      most = lo + step < most ? lo + step : most;
    }
    pair = lo;
    const long long ahead = lane_value(work, 0), each = lane_value(work, 1) - ahead;
    base += n * ahead;
    h = small_quotient(from_work - base, each);
    base += h * each;
    in_chunk = n - h;
    h += chunk_first;
    tile = tiles - 1 - pair;
    const long long later = START + prompt_keys(P, seq, tile).count;
    if (tile != pair && from_work >= base + later) { base += later; tile = pair; }
    base = uniform(base + START);
    h = __builtin_amdgcn_readfirstlane(h); tile = __builtin_amdgcn_readfirstlane(tile); in_chunk = __builtin_amdgcn_readfirstlane(in_chunk); chunk_first = __builtin_amdgcn_readfirstlane(chunk_first);
    keys = prompt_keys(P, seq, tile);
    part();
    return mine_first() || next(P);
  }
  // the sequence's tiles and chunks, from its work for one head
  __device__ __forceinline__ void enter(const PromptParams &P, long long per_head) {
    tiles = prompt_tiles(P, seq);
    const float n = (float)((tiles + 1) / 2) * (float)per_share / (float)per_head;           // (rounded as it may be: the same in every workgroup)
    chunk_heads = __builtin_amdgcn_readfirstlane(n < 1.5f ? 1 : n >= (float)P.heads ? P.heads : (int)(n + 0.5f));
  }
  // work of the first n pairs of one head
  __device__ __forceinline__ long long pairs_work(const PromptParams &P, long long per_head, int n) const {
    return per_head - prompt_work<START>(P, seq, tiles - n) + prompt_work<START>(P, seq, n < tiles - n ? n : tiles - n);
  }
  // the workgroup's keys of the present tile: whole stages from the tile's first key on, each of the share that its last key falls into
  __device__ __forceinline__ void part() {
    auto stages = [&](long long o) { return o <= 0 ? 0 : o >= keys.count ? keys.count : (int)o / UNIT * UNIT; };
    k_from = stages(from_work - base); k_to = stages(end - base);
  }
  // a tile without keys is that of the share that its beginning falls into
  __device__ __forceinline__ bool mine_first() const { return keys.count > 0 ? k_from < k_to : from_work <= base - START && base - START < end; }
  // on to the next tile with keys (or rows to clear) of this workgroup
  __device__ __forceinline__ bool next(const PromptParams &P) {
    do {
      base += keys.count + START;
      if (base - START >= end) return false;
      if (tile > pair) {
        tile = pair;
      } else {
        ++h;
        if (--in_chunk == 0) {
          h = chunk_first;
          if (++pair == (tiles + 1) / 2) {
            pair = 0;
            h = chunk_first += chunk_heads;
            if (h >= P.heads) {
              h = chunk_first = 0;
              do {
                if (++s >= P.n_seqs) return false;
                seq = prompt_seq(P, s);
              } while (seq.n == 0);
              enter(P, prompt_work<START>(P, seq, prompt_tiles(P, seq)));
            }
          }
          in_chunk = P.heads - h < chunk_heads ? P.heads - h : chunk_heads;
        }
        tile = tiles - 1 - pair;
      }
      keys = prompt_keys(P, seq, tile);
      part();
    } while (!mine_first());
    return true;
  }
  // the workgroup has all of the present tile; it has its first keys
  __device__ __forceinline__ bool whole() const { return k_from == 0 && k_to == keys.count; }
  __device__ __forceinline__ bool first() const { return k_from == 0; }
  // shares that have stages of the present tile
  __device__ __forceinline__ int sharers() const {
    const int one = keys.count < UNIT ? keys.count : UNIT;
    return (int)((base + keys.count - 1) / per_share - (base + one - 1) / per_share + 1);
  }
};

// A row of a tile: its token and query head; false: there is none.
__device__ __forceinline__ bool prompt_row(const PromptParams &P, const PromptSeq &q, int tile, int h, int r, int &token, int &head) {
  const int j = r / P.tile_group, g = r - j * P.tile_group, kv = h / P.head_tiles, g0 = (h - kv * P.head_tiles) * P.tile_group;
  token = tile * P.tile_tokens + j;
  head = kv * P.group + g0 + g;
  return j < P.tile_tokens && token < q.n && g0 + g < P.group;
}

// What a tile costs beside its keys, in keys.  With 256 rows it is 5 to 6 us (the run's next tile 1, its queries 1, the output 2, the
// first slots' products with nothing beside them 2); 128 in place of 256: windows of 1024 keys, heads of 256, 448 us instead of 428,
// 256 prompts of 64 tokens 27 instead of 21; 512 the same as 256 within 1 %.  Up to 16 rows: 32 against 128 is 14.8 us against 16.5
// for 8 tokens over 1000 keys and 51.7 against 51.3 for 128 over 500.
template <int ROWS> constexpr int PROMPT_START = ROWS == 16 ? 32 : 256;

// ---- up to 16 rows per tile: single tokens and the like over long caches.  Four wavefronts, each its own 32 of 128 keys,
// operands straight from memory into registers (the products and the way of V's operand are those of tree_attention_kernel).
// Bound by HBM: 64 sequences with one token each, 64 query and 8 key heads of 128, 0 .. 8191 keys: 1.08 GB in 209 us, 5.2 TB/s (a large
// copy reaches 5.0, a read alone 6).
template <int DT, int DP, bool FULL>
__global__ __launch_bounds__(ATT_THREADS) void prompt_rows_kernel(const PromptParams P) {
  constexpr int WK = ATT_THREADS / 64, UNIT = ATT_KEYS * WK, ROWS = 16, START = PROMPT_START<16>;
  constexpr int KS = DP / 32, VE = DP == 64 ? 4 : 8, NC = DP / (16 * VE), NF = NC * VE, VW = VE / 2, OP = DP + 4;
  constexpr float LIFT = DT == DT_F16 ? 32768.0f : 1.0f;           // (as there: fp16's small numbers)
  constexpr uint32_t ONES = DT == DT_F16 ? 0x3c003c00u : 0x3f803f80u;
  __shared__ __attribute__((aligned(16))) float merge_o[WK * 16 * OP];
  __shared__ float merge_ml[2 * WK * 16];
  __shared__ long long scan[ATT_THREADS / 64];
  __shared__ long long found[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, quarter = lane >> 4;
  const int D = FULL ? DP : P.head_dim;
  const int share = run_tile_of(blockIdx.x, P.n_shares);

  PromptRun<UNIT, START, ATT_THREADS> run;
  if (tid == 0) P.joins[share] = make_int4(-1, 0, 0, 0);
  if (!run.begin(P, share, scan, found)) return;                   // (the same in every thread)
  do {
    const PromptSeq seq = run.seq;
    const int s = run.s, h = run.h, tile = run.tile, kv = h / P.head_tiles;
    int token, head;
    const bool row = prompt_row(P, seq, tile, h, col, token, head);  // this lane's row
    u32x4_t qf[KS];
    {
      const uint16_t *qp = P.q + (long long)(seq.row0 + token) * P.ldq + (long long)head * D + quarter * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qf[ks] = u32x4_t{0u, 0u, 0u, 0u};
        if (row && (FULL || ks * 32 + quarter * 8 < D)) qf[ks] = *reinterpret_cast<const u32x4_t *>(qp + ks * 32);
      }
    }
    f32x4_t o[NF], l = {0.0f, 0.0f, 0.0f, 0.0f};
    float m = -__builtin_inff();
    const u32x4_t ones = {ONES, ONES, ONES, ONES};
#pragma unroll
    for (int f = 0; f < NF; ++f) o[f] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    // the keys that this lane's row sees: [low, high]; those that every row of the tile sees: [all_low, all_high]
    const int place = seq.keys - seq.n + token, low = place - P.left, high = row ? place + P.right : -1;
    const int t_last = (tile + 1) * P.tile_tokens < seq.n ? (tile + 1) * P.tile_tokens - 1 : seq.n - 1;
    const int all_low = seq.keys - seq.n + t_last - P.left, all_high = seq.keys - seq.n + tile * P.tile_tokens + P.right;

    const char *kh = reinterpret_cast<const char *>(P.k + (long long)kv * D) + (uint64_t)seq.key0 * P.ldk;
    const char *vh = reinterpret_cast<const char *>(P.v + (long long)kv * D) + (uint64_t)seq.key0 * P.ldv;
    const int k_last = run.keys.first + run.k_to;
    for (int k0 = run.keys.first + run.k_from + wave * ATT_KEYS; k0 < k_last; k0 += UNIT) {
      const uint32_t live = seq.keys - k0 >= 32 ? 0xffffffffu : (1u << (seq.keys - k0)) - 1u;        // the keys that exist
      const bool whole = live == 0xffffffffu;
      const char *kp = kh + (uint64_t)(uint32_t)k0 * P.ldk, *vp = vh + (uint64_t)(uint32_t)k0 * P.ldv;
      auto held = [&](int x) { return whole || x < seq.keys - k0 ? x : seq.keys - k0 - 1; };          // (rows behind the last are not read)
      u32x4_t kf[2][KS];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const char *kr = kp + (uint64_t)(uint32_t)held(16 * u + col) * P.ldk + quarter * 16;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          kf[u][ks] = u32x4_t{0u, 0u, 0u, 0u};
          if (FULL || ks * 32 + quarter * 8 < D) kf[u][ks] = *reinterpret_cast<const u32x4_t *>(kr + ks * 64);
        }
      }
      uint32_t vw[NC][8][VW];                    // [piece][key 4 u + i of the lane][word]
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const char *vr = vp + (uint64_t)(uint32_t)held(16 * (x / 4) + 4 * quarter + x % 4) * P.ldv + col * VE * 2;
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
      const bool masked = !whole || k0 + 31 > all_high || k0 < all_low;
      uint32_t sees = 0xffffffffu;               // of the 32 keys
      bool odd_v = false;                        // a value that is infinite or NaN beside rows that do not see it
      if (masked) {
#pragma unroll
        for (int x = 0; x < 8; ++x) {
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
        const int up = high - k0 + 1, down = low - k0;
        sees = (up >= 32 ? 0xffffffffu : up <= 0 ? 0u : (1u << up) - 1u) & (down <= 0 ? 0xffffffffu : down >= 32 ? 0u : 0xffffffffu << down) & live;
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
      const float base = m == -__builtin_inff() ? 0.0f : m;        // (a row that has seen no key yet)
#pragma unroll
      for (int x = 0; x < 8; ++x) p[x] = att_exp2(p[x] - base) * LIFT;
      // the probabilities, at most LIFT, as the 16-bit operand of the second product: each is off by at most half a step of the
      // type, which is what the output's own rounding is off by; the sum is that of the rounded ones
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
          const uint16_t *vr = reinterpret_cast<const uint16_t *>(vp + (uint64_t)(uint32_t)kk * P.ldv);
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
    const bool whole = run.whole();
    const long long which = 2LL * share + (run.first() ? 1 : 0);    // (a tile that begins here is the last of the run, one that does not the first)
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
      int t, hh;
      if (!prompt_row(P, seq, tile, h, rr, t, hh) || (!FULL && d >= D)) continue;
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
      if (whole) {
        uint16_t *op = P.out + (long long)(seq.row0 + t) * P.ldo + (long long)hh * D + d;
        const float inv = ll > 0.0f || ll != ll ? 1.0f / ll : 0.0f;               // (no key seen: zeros)
        uint32_t w[VW];
#pragma unroll
        for (int i = 0; i < VW; ++i) w[i] = pack2<DT>(y[2 * i] * inv, y[2 * i + 1] * inv);
        if constexpr (VE == 8) *reinterpret_cast<u32x4_t *>(op) = u32x4_t{w[0], w[1], w[2], w[3]};
        else *reinterpret_cast<uint2 *>(op) = make_uint2(w[0], w[1]);
      } else {
        float *pp = P.part + (which * ROWS + rr) * DP + d;
#pragma unroll
        for (int i = 0; i < VE; i += 4) *reinterpret_cast<f32x4_t *>(pp + i) = f32x4_t{y[i], y[i + 1], y[i + 2], y[i + 3]};
        if (d == 0) P.part_ml[which * ROWS + rr] = make_float2(mm, ll);
      }
    }
    if (!whole && run.first() && tid == 0) P.joins[share] = make_int4(s, h, tile, run.sharers());
  } while (run.next(P));
}

// ---- more rows: WAVES wavefronts with 32 rows each share the keys, SLOT at a time, through a ring of four slots in LDS.
//
// Scores are computed as S^T = K Q^T, so that a lane has 16 scores of one row, which rounded to the type are the operand of
// O^T += V^T P^T as they are; V's operand is read transposed.  A slot's rows go from memory to LDS without registers, three slots ahead,
// across the ends of tiles, with one barrier a slot.  A row's reference is its first maximum, moved to where the powers of two use
// the type's range, and changed only when a probability gets large: most turns (32 keys) neither take a maximum nor rescale.
//
// Bound by the issue of one wavefront's instructions: a turn of heads of 128 has 16 products of 32 cycles and 78 vector instructions, of which 16
// are exponentials, and a product hides about five of them (three beside an exponential).  So the products of the turn before run beside the
// probabilities, the next scores beside the sum and the reads of V, in a fixed order, and registers hold 32 rows: with 64 rows per
// wavefront (half the reads from LDS) 970 TFLOP/s, with two groups of wavefronts in opposite halves of a turn 950, both when this form was at 1015.
//   one prompt of 16384 tokens, 64 query and 8 key heads of 128, bf16     4.40 TFLOP    4.0 ms    1100 TFLOP/s (a large library product: 1210)
//   16 of 1344 .. 2500, 32 heads of 128, fp16                             0.53          0.77      684
//   4 of 3454 .. 6000, windows of 1024, 16 query and 8 key heads of 256   0.30          0.46      661
//   24 images of 532 .. 1024 patches, 16 heads of 80, fp16                0.067         0.16      420
// In the first the matrix units are busy for 53 % of the cycles and the clock goes down to 1.8 to 2 GHz: at that point power takes part in the bound.
// In the others tiles have few keys: PROMPT_START, what a tile costs beside them, is 18 to 23 % of the work.  Heads of 80 have 11 products a turn (352
// cycles) for the same vector instructions (about 500): the matrix units are busy for 26 % of the cycles.
// KS: 16-feature steps of the first product (padded head dimension 16 KS); PITCH: features of a row in LDS.
template <int KS_, int WAVES_> struct PromptTile {
  static constexpr int KS = KS_, WAVES = WAVES_;
  static constexpr int PITCH = KS <= 4 ? 64 : KS <= 8 ? 128 : 256;
  static constexpr int NF = (KS + 1) / 2;        // 32-feature blocks of the output
  static constexpr int SLOT = PITCH == 256 ? 32 : 64;
  static constexpr int THREADS = 64 * WAVES, ROWS = 32 * WAVES, RING = 4;
  static constexpr int ROWB = 2 * PITCH, BUF = SLOT * ROWB, LDS = RING * 2 * BUF;
  static constexpr int COLS = 32 * NF;           // columns of a partial output
};
constexpr int PROMPT_UNIT = 64;                  // keys of two steps of a wavefront

__device__ const u32x4_t prompt_zeros[32] = {};  // a row of zeros

// The 16-byte pieces of a row in LDS are XORed with a number of the row's.  K: 32 rows at one piece are read 8 at a time, which
// then cover all banks.  V: a transposing read takes 32 bytes of four neighbouring rows by 16 lanes, and with them in four different
// groups of four pieces all banks are covered too.
template <int PITCH> __device__ __forceinline__ int prompt_swizzle_k(int row) { return PITCH == 64 ? (row >> 1) & 7 : row & 15; }
template <int PITCH> __device__ __forceinline__ int prompt_swizzle_v(int row) {
  return PITCH == 64 ? (row & 2) << 1 : (row & 3) << 2 | ((row >> 2) & 3);
}

// c + both 16-bit values of a word
template <int DT> __device__ __forceinline__ float add_pair(uint32_t w, float c) {
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (DT == DT_F16) return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2_t, w), __builtin_bit_cast(f16x2_t, 0x3c003c00u), c, false);
  else return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w), __builtin_bit_cast(bf16x2_t, 0x3f803f80u), c, false);
#else
  (void)w;
  return c;
#endif
}

// load_to_lds with LDS addresses as numbers
__device__ __forceinline__ void load_to_lds_at(const void *from, uint32_t offset, uint32_t to) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(from) : "memory", "m0");
#else
  (void)from; (void)offset; (void)to;
#endif
}
__device__ __forceinline__ void load_to_lds_at(const void *from, uint32_t to) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory", "m0");
#else
  (void)from; (void)to;
#endif
}
// pairs of 16-bit numbers: the larger, the smaller, the product's low halves, the difference or 0
typedef unsigned short pair_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t larger_pair(uint32_t a, uint32_t b) { return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(pair_t, a), __builtin_bit_cast(pair_t, b))); }
__device__ __forceinline__ uint32_t smaller_pair(uint32_t a, uint32_t b) { return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(pair_t, a), __builtin_bit_cast(pair_t, b))); }
__device__ __forceinline__ uint32_t times_pair(uint32_t a, uint32_t b) { return __builtin_bit_cast(uint32_t, __builtin_bit_cast(pair_t, a) * __builtin_bit_cast(pair_t, b)); }
__device__ __forceinline__ uint32_t minus_pair(uint32_t a, uint32_t b) { return __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(__builtin_bit_cast(pair_t, a), __builtin_bit_cast(pair_t, b))); }

// the upper half wave's a and the lower half's b change places
__device__ __forceinline__ void halves_swap(uint32_t &a, uint32_t &b) {
#if defined(__HIP_DEVICE_COMPILE__)
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0]; b = r[1];
#endif
}

template <int DT, int KS, int WAVES, bool FULL>
__global__ __launch_bounds__(64 * WAVES, WAVES / 4) void prompt_tile_kernel(const PromptParams P) {
  using C = PromptTile<KS, WAVES>;
  constexpr int ROWS = C::ROWS, SLOT = C::SLOT, THREADS = C::THREADS, NF = C::NF, ROWB = C::ROWB, BUF = C::BUF, START = PROMPT_START<ROWS>;
  constexpr int CH = C::PITCH / 8;               // 16-byte pieces of a row
  constexpr int WROWS = SLOT / WAVES;            // rows of K (of V) that a wavefront loads of a slot
  constexpr int RPI = 64 / CH, NL = WROWS / RPI; // rows of one load instruction, load instructions
  constexpr bool LEAVE = SLOT == 64;             // turns in which the wavefront's rows see nothing are left to the others (heads of 256 have no registers for it)
  constexpr float REF = DT == DT_F16 ? -12.0f : 16.0f, NONE = 3.402823466e38f, FAR = 16777216.0f;
  static_assert(NL * RPI == WROWS, "whole load instructions");
  extern __shared__ __attribute__((aligned(16))) unsigned char prompt_smem[];   // [RING][K, V][SLOT][ROWB]
  __shared__ long long scan[THREADS / 64];
  __shared__ long long found[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int D = FULL ? 16 * KS : P.head_dim;
  const int share = run_tile_of(blockIdx.x, P.n_shares);
  // Where the wavefront is in its run, and where its loads are, ahead of that: in LDS, so that the loop has the scalar registers.
  using Run = PromptRun<PROMPT_UNIT, START, THREADS>;
  __shared__ Run kept[2][WAVES];
  {
    Run run;
    if (tid == 0) P.joins[share] = make_int4(-1, 0, 0, 0);
    if (!run.begin(P, share, scan, found)) return;                 // (the same in every thread)
    kept[0][wave] = run; kept[1][wave] = run;
  }
  auto advance = [&](int which) __attribute__((always_inline)) -> bool {
    Run run = kept[which][wave];
    const bool more = __builtin_amdgcn_readfirstlane(run.next(P));
    kept[which][wave] = run;
    return more;
  };
  auto scalar = [](int x) { return __builtin_amdgcn_readfirstlane(x); };

  // byte offset of this lane's operand of K in 32 rows, for the first step; for step ks its bits of 32 ks are the other way
  const int kbase = col * ROWB + ((half ^ prompt_swizzle_k<C::PITCH>(col)) * 16);
  // row (of 16: keys 4 half + ... and, 8 further, the same) that this lane addresses in a transposing read of V, and its 8 bytes there
  const int vrow = 4 * half + ((lane & 15) >> 2), vpiece = (((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) ^ prompt_swizzle_v<C::PITCH>(vrow);
  const int vbase = vrow * ROWB + (lane & 1) * 8;

  // The slots to be loaded run ahead of those in use, over the ends of tiles.  Of the next one: the wavefront's first row of K and of
  // V, and how far behind it (in bytes) the sequence's last key is.  Rows behind the last key are that key's again: nothing sees them.
  const char *kr = reinterpret_cast<const char *>(prompt_zeros), *vr = kr;
  uint32_t k_most = 0, v_most = 0;
  int steady = 0, after = -1;                    // slots to come that only move on; where in the tile's keys the one behind them begins
  bool over = false;
  auto another_slot = [&]() __attribute__((always_inline)) {
    steady = 0;
    if (over) return;
    if (after < 0) after = scalar(kept[1][wave].k_from);
    // (a tile's slots are those of whole units; one without keys has none)
    auto units_end = [&] { return (scalar(kept[1][wave].k_to) + PROMPT_UNIT - 1) / PROMPT_UNIT * PROMPT_UNIT; };
    while (after >= units_end()) {
      if (!advance(1)) {                         // no slot is left: rows of zeros, which nothing reads
        over = true;
        kr = vr = reinterpret_cast<const char *>(prompt_zeros);
        k_most = v_most = 0;
        return;
      }
      after = scalar(kept[1][wave].k_from);
    }
    const Run &at = kept[1][wave];
    const int kv = scalar(at.h) / P.head_tiles, keys = scalar(at.seq.keys), k0 = scalar(at.keys.first) + after + WROWS * wave;
    const int rest = keys - k0;                  // keys from the wavefront's first row on
    const uint32_t row0 = scalar(at.seq.key0) + (rest > 0 ? k0 : keys - 1);
    kr = reinterpret_cast<const char *>(P.k + (long long)kv * D) + (uint64_t)row0 * P.ldk;
    vr = reinterpret_cast<const char *>(P.v + (long long)kv * D) + (uint64_t)row0 * P.ldv;
    k_most = v_most = 0xffffffffu;
    int here = 1;
    if (rest < WROWS) {
      const uint32_t last = rest > 0 ? rest - 1 : 0;
      k_most = last * P.ldk; v_most = last * P.ldv;
    } else {
      const int whole = (rest - WROWS) / SLOT + 1, left = (units_end() - after) / SLOT;
      here = whole < left ? whole : left;
    }
    steady = here - 1;
    after += here * SLOT;
  };
  auto next_slot = [&]() __attribute__((always_inline)) {
    if (__builtin_expect(steady > 0, 1)) {
      --steady;
      kr += (uint64_t)SLOT * P.ldk; vr += (uint64_t)SLOT * P.ldv;
    } else {
      another_slot();
    }
  };
  // This lane's part of a load instruction: its row (in bytes) and its piece; those of instruction i are RPI i rows further on.
  const uint32_t k_row = (lane / CH) * P.ldk, v_row = (lane / CH) * P.ldv;
  const uint32_t k_off = ((lane % CH) ^ prompt_swizzle_k<C::PITCH>(WROWS * wave + lane / CH)) * 16, v_off = ((lane % CH) ^ prompt_swizzle_v<C::PITCH>(WROWS * wave + lane / CH)) * 16;
  const uint32_t ring = lds_at(prompt_smem) + wave * WROWS * ROWB;             // the wavefront's rows of the ring's first place
  // The 2 NL load instructions that bring its rows into place b of the ring: as many whatever keys there are, so that the waits
  // below can count them.
  auto issue = [&](int b) __attribute__((always_inline)) {
    const char *ks = kr, *vs = vr;
    settled(ks, vs);
#pragma unroll
    for (int i = 0; i < 2 * NL; ++i) {
      const bool v = i % 2;
      const uint32_t place = ring + b * 2 * BUF + (v ? BUF : 0) + i / 2 * 1024, ld = v ? P.ldv : P.ldk, most = v ? v_most : k_most;
      const uint32_t piece = (v ? v_off : k_off) ^ ((v ? prompt_swizzle_v<C::PITCH>(RPI * (i / 2)) : prompt_swizzle_k<C::PITCH>(RPI * (i / 2))) * 16);
      uint32_t at = (v ? v_row : k_row) + RPI * (i / 2) * ld;
      at = (at < most ? at : most) + piece;
      if constexpr (FULL && 16 * KS == C::PITCH) load_to_lds_at(v ? vs : ks, at, place);
      else load_to_lds_at((int)piece < 2 * D ? (v ? vs : ks) + at : reinterpret_cast<const char *>(prompt_zeros), place);          // features behind the head's are zeros
    }
  };
  auto read_k = [&](const unsigned char *kb, u32x4_t (&kf)[KS]) __attribute__((always_inline)) {          // of the 32 keys at kb
    int kx = kbase;
    asm volatile("" : "+v"(kx));                 // (what is made of it is not kept through the loop)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kf[ks] = *reinterpret_cast<const u32x4_t *>(kb + (kx ^ (ks * 32)));
  };

  for (int i = 0; i < 3; ++i) { next_slot(); issue(i); }
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NL) : "memory");
  __builtin_amdgcn_s_barrier();                  // slots 0 and 1 have landed
  asm volatile("" ::: "memory");
  int b = 0;
  // The present tile: the lane's row (its token and head of the tile are always the same), its queries and the keys that it sees.
  const int row_token = (wave * 32 + col) / P.tile_group, row_head = (wave * 32 + col) % P.tile_group;
  PromptSeq seq;
  int h, tile, low, high, k_first, k_last;
  bool row;
  long long row_at, head_at;                     // the row's token, and its head's first feature
  u32x4_t qf[KS];
  auto open_tile = [&]() __attribute__((always_inline)) {
    const Run &at = kept[0][wave];
    seq = {scalar(at.seq.row0), scalar(at.seq.n), scalar(at.seq.key0), scalar(at.seq.keys)};
    h = scalar(at.h); tile = scalar(at.tile);
    k_first = scalar(at.keys.first + at.k_from); k_last = scalar(at.keys.first + at.k_to);
    const int kv = h / P.head_tiles, g0 = (h - kv * P.head_tiles) * P.tile_group, token = tile * P.tile_tokens + row_token;
    row = row_token < P.tile_tokens && token < seq.n && g0 + row_head < P.group;
    row_at = seq.row0 + token;
    head_at = (long long)(kv * P.group + g0 + row_head) * D;
    const uint16_t *qp = P.q + row_at * P.ldq + head_at + half * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qf[ks] = u32x4_t{0u, 0u, 0u, 0u};
      if (row && (FULL || ks * 16 + half * 8 < D)) qf[ks] = *reinterpret_cast<const u32x4_t *>(qp + ks * 16);
    }
    const int place = seq.keys - seq.n + token;
    low = place - P.left;
    high = row ? place + P.right : -1;
    high = high < seq.keys - 1 ? high : seq.keys - 1;
  };
  open_tile();
  bool more;
  do {
    // The queries are waited for here, with what is under way to LDS: left to the compiler, which does not know of the loads in
    // assembly, the wait stands ahead of every use in the loop below, and there it is one for all rows of K and V under way.  (The
    // output's stores are waited for too; a wait ahead of them in its place measured the same.)
    __builtin_amdgcn_s_waitcnt(0x0f70);          // vmcnt(0)
    // keys that every row of the wavefront sees (rows that are none see nothing and need no mask)
    const int w0 = wave * 32 / P.tile_group, w1 = (wave * 32 + 31) / P.tile_group, t_first = tile * P.tile_tokens + w0;
    int t_last = tile * P.tile_tokens + (w1 < P.tile_tokens ? w1 : P.tile_tokens - 1);
    t_last = t_last < seq.n ? t_last : seq.n - 1;
    int all_high = seq.keys - seq.n + t_first + P.right;
    const int all_low = seq.keys - seq.n + t_last - P.left;
    all_high = all_high < seq.keys - 1 ? all_high : seq.keys - 1;
    // Keys that some row of it sees are in [some_low, some_high] (none: it has no rows).  Turns beyond are left out but for one on
    // either side, in which nothing is seen: the last adds up the values of the turn before.
    const int some_low = seq.keys - seq.n + t_first - P.left, some_high = w0 < P.tile_tokens && t_first < seq.n ? seq.keys - seq.n + t_last + P.right : -PROMPT_FAR;
    f32x16_t o[NF];
    float l[2];                                  // two parts of the sum over the lane's own keys: the wave's other half has the rest
    float ref;                                   // -m; NONE, fp32's largest number, where a row has seen no key yet: any score but minus infinity then makes an infinity
    bool far_off = false;                        // some row's reference is FAR or more in size
    // A turn of a wavefront (32 keys): the scores become probabilities while the matrix unit adds up the values of the turn before;
    // then the scores of the next turn are formed while the values of this one are read.
    u32x4_t kf[KS], vf[NF][2], pf[2][2];         // pf: probabilities of the turn before, of this one
    f32x16_t x;                                  // scores
    l[0] = l[1] = 0.0f;
    ref = NONE;
    pf[0][0] = pf[0][1] = pf[1][0] = pf[1][1] = u32x4_t{0u, 0u, 0u, 0u};
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[f][i] = 0.0f;
#pragma unroll
    for (int f = 0; f < NF; ++f) vf[f][0] = vf[f][1] = u32x4_t{0u, 0u, 0u, 0u};
    auto scores = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = 0.0f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        x = mfma32<DT>(kf[ks], qf[ks], x);
    };
    // Values that are infinite or NaN among the 32 keys from k0 on, some of which some row does not see: 0 x infinity is no number.  They
    // are taken out of the operand, and where a row sees one, its product with the row's probability is added to the row's output: an
    // infinite value's is no number where the probability is 0, as in turns that every row sees, and what the value is elsewhere.
    auto odd_values = [&](int k0, const u32x4_t (&prob)[2]) __attribute__((always_inline)) {
      constexpr uint32_t INF = DT == DT_F16 ? 0x7c007c00u : 0x7f807f80u, ONE = DT == DT_F16 ? 0x3c00u : 0x3f80u;
      uint32_t most = 0;
#pragma unroll
      for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
          for (int w = 0; w < 4; ++w) most = larger_pair(most, vf[f][kk][w] & 0x7fff7fffu);
      if (!__any(not_finite<DT>(most))) return;
      u32x4_t see[2];                            // ones for the keys that the lane's rows see, as the operand of probabilities
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const int key = k0 + 8 * (i / 4) + 4 * half + i % 4;
        see[i / 8][(i % 8) / 2] = (key >= low && key <= high ? ONE : 0u) | (key + 1 >= low && key + 1 <= high ? ONE << 16 : 0u);
      }
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        asm volatile("" : "+v"(vf[f][0]), "+v"(vf[f][1]));         // (nothing of this is kept from the test above, or for the next block)
#pragma unroll 1
        for (int kind = 0; kind < 4; ++kind) {   // infinity, minus infinity, NaN, an infinity of either sign (or NaN) beside a probability of 0
          const uint32_t add = kind == 0 ? 0x7f800000u : kind == 1 ? 0xff800000u : 0x7fc00000u;
          const uint32_t hide = kind >= 2 ? 0x7fff7fffu : 0xffffffffu, other = kind == 0 ? INF : kind == 1 ? INF | 0x80008000u : 0u;
          const uint32_t under = kind == 2 ? INF : INF - 0x00010001u;
          const uint32_t all = kind == 2 ? 0xffffffffu : 0u, turned = kind == 3 ? 0xffffffffu : 0u;
          f32x16_t n;
#pragma unroll
          for (int i = 0; i < 16; ++i) n[i] = 0.0f;
#pragma unroll
          for (int kk = 0; kk < 2; ++kk) {
            u32x4_t one, mine;
#pragma unroll
            for (int w = 0; w < 4; ++w) {        // (arithmetic on pairs: 1 where it is one of the kind)
              const uint32_t v = (vf[f][kk][w] & hide) ^ other;
              one[w] = times_pair(kind >= 2 ? smaller_pair(minus_pair(v, under), 0x00010001u) : smaller_pair(v, 0x00010001u) ^ 0x00010001u, ONE * 0x00010001u);
              const uint32_t some = times_pair(smaller_pair(prob[kk][w] & 0x7fff7fffu, 0x00010001u), 0xffffffffu);       // (all ones where the probability is not 0)
              mine[w] = see[kk][w] & ((some ^ turned) | all);
            }
            n = mfma32<DT>(one, mine, n);
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) {       // (n: how many the row sees)
            const uint32_t some = __float_as_uint(n[i]) < 1u ? __float_as_uint(n[i]) : 1u;
            o[f][i] += __uint_as_float((0u - some) & add);
          }
        }
        asm volatile("" : "+v"(vf[f][0]), "+v"(vf[f][1]));
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t odd = smaller_pair(minus_pair(vf[f][kk][w] & 0x7fff7fffu, INF - 0x00010001u), 0x00010001u);
            vf[f][kk][w] &= ~times_pair(odd, 0xffffffffu);
          }
      }
    };
    if (k_first < k_last) {
      read_k(prompt_smem + b * 2 * BUF, kf);
      scores();
    }
    bool hidden = false;                         // of the keys of the turn before, some row does not see some
    for (int k0 = k_first; k0 < k_last; k0 += PROMPT_UNIT) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        if (c * 32 % SLOT == 0) {
          // my rows of the next slot have landed, and what I read of the slot before has been read ...
          asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * NL) : "memory");
          __builtin_amdgcn_s_barrier();          // ... and everybody's
          asm volatile("" ::: "memory");
          next_slot();
          issue((b + 3) & 3);
        }
        const unsigned char *vb = prompt_smem + b * 2 * BUF + BUF + c * 32 % SLOT * ROWB;
        if ((c + 1) * 32 % SLOT == 0) b = (b + 1) & 3;
        const unsigned char *kb = prompt_smem + b * 2 * BUF + (c + 1) * 32 % SLOT * ROWB;          // of the 32 keys after these
        const int k = k0 + 32 * c;
        if (LEAVE && (k > some_high + 32 || k + 63 < some_low)) continue;
        const bool masked = k + 31 > all_high || k < all_low;
        if (__builtin_expect(masked || hidden, 0)) {
          if (hidden) odd_values(k - 32, pf[1 - c]);
          if (masked) {
            const int up = high - k - 4 * half, down = low - k - 4 * half;
#pragma unroll
            for (int i = 0; i < 16; ++i) {     // key 8 (i / 4) + 4 half + i % 4 of the 32
              const int at = 8 * (i / 4) + i % 4;
              if (at > up || at < down) x[i] = -__builtin_inff();
            }
          }
        }
        hidden = masked;
        u32x4_t (&p)[2] = pf[c], (&before)[2] = pf[1 - c];
        uint32_t any = 0;
        // Probabilities, rounded to the type: off by at most half a step, which is what the output's own rounding is off by.  Two at a
        // time, in three steps (the scaled score, its power, the rounding) of which each is done beside the others' next two.
        float e[16];
        auto scale = [&](int i) __attribute__((always_inline)) { e[i] = fmaf(x[i], P.scale2, ref); e[i + 1] = fmaf(x[i + 1], P.scale2, ref); };
        auto power = [&](int i) __attribute__((always_inline)) { e[i] = att_exp2(e[i]); e[i + 1] = att_exp2(e[i + 1]); };
        auto round = [&](int i) __attribute__((always_inline)) {
          p[i / 8][(i % 8) / 2] = pack2<DT>(e[i], e[i + 1]);
          if (i % 4 == 2) any = att_larger<DT>(any, p[i / 8][(i % 8) / 2 - 1], p[i / 8][(i % 8) / 2]);
        };
        // ---- beside them the products that add up the values of the turn before (each hides five vector instructions, an exponential
        // counting for two), and the reads of the next scores' operands
        int kx = kbase, vx = vbase, vz = vpiece;
        asm volatile("" : "+v"(kx));             // (what is made of it is not kept through the loop)
        __builtin_amdgcn_sched_barrier(0);
        constexpr int N1 = 2 * NF, STEPS = 10, N3 = (2 * KS + 2) / 3;    // (the values' last reads have a third of the products to come back)
#pragma unroll
        for (int i = 0; i < N1; ++i) {
          o[i % NF] = mfma32<DT>(vf[i % NF][i / NF], before[i / NF], o[i % NF]);
#pragma unroll
          for (int ks = i * KS / N1; ks < (i + 1) * KS / N1; ++ks) kf[ks] = *reinterpret_cast<const u32x4_t *>(kb + (kx ^ (ks * 32)));
#pragma unroll
          for (int j = i * STEPS / N1; j < (i + 1) * STEPS / N1; ++j) {
            if (j < 8) scale(2 * j);
            if (j >= 1 && j <= 8) power(2 * j - 2);
            if (j >= 2) round(2 * j - 4);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        if (__builtin_expect(__any(att_large<DT>(any)) || far_off, 0)) {
          float top = x[0];
#pragma unroll
          for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
          top = fmaxf(top, __shfl_xor(top, 32, 64)) * P.scale2;
          // The fused product above has more bits than the rounded one that the reference is made of: beside a reference of 2^24 (FAR)
          // the difference is a factor of up to 2, beside one of 2^31 an infinity or nothing.  From FAR on the wavefront rounds the
          // products, takes the maximum of every 32 keys, and a row's largest probability is 1.
          const bool seen = top != -__builtin_inff(), far = seen && fabsf(top) >= FAR;
          far_off |= __any(far) != 0;
          const float ref_new = !seen ? ref : fminf(ref, far ? -top : -(top + REF));
          const float a = att_exp2(ref_new - ref);         // (0 from NONE on)
          ref = ref_new;
          l[0] *= a; l[1] *= a;
#pragma unroll
          for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[f][i] *= a;
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            if (far_off) {
              float t[2];
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                t[j] = x[i + j] * P.scale2;
                asm volatile("" : "+v"(t[j])); // (not fused with the sum)
              }
              p[i / 8][(i % 8) / 2] = pack2<DT>(att_exp2(t[0] + ref), att_exp2(t[1] + ref));
            } else {
              scale(i); power(i); round(i);
            }
          }
        }
        // ---- the scores of the next turn; beside them the values of this turn are read, and the sum
        asm volatile("" : "+v"(vx), "+v"(vz));
        auto read_v = [&](int i) __attribute__((always_inline)) {  // keys 16 kk + 8 u + vrow: their swizzle is that of vrow with the bits of 8 u the other way
          const int f = i / 4, kk = i / 2 % 2, u = i % 2;
          const uint2 v = read_transposed(vb + (16 * kk + 8 * u) * ROWB + vx + (((f * 4) ^ vz ^ prompt_swizzle_v<C::PITCH>(8 * u)) * 16));
          vf[f][kk][2 * u] = v.x; vf[f][kk][2 * u + 1] = v.y;
        };
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 0.0f;
#pragma unroll
        for (int n = 0; n < KS; ++n) {
          x = mfma32<DT>(kf[n], qf[n], x);
#pragma unroll
          for (int i = n * 4 * NF / N3; i < (n + 1) * 4 * NF / N3 && i < 4 * NF; ++i) read_v(i);
#pragma unroll
          for (int i = n * 8 / KS; i < (n + 1) * 8 / KS; ++i) l[i % 2] = add_pair<DT>(p[i / 4][i % 4], l[i % 2]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    const int k_end = k_first + (k_last - k_first + PROMPT_UNIT - 1) / PROMPT_UNIT * PROMPT_UNIT - 32;        // of the last turn
    const bool rest = k_first < k_last && (!LEAVE || k_end <= some_high);        // the last turn's values are to be added
    if (rest && hidden) odd_values(k_end, pf[1]);

    // ---- out: to the rows, where this workgroup had all their keys, else to the workspace; the next tile's queries are asked for
    // ahead of that
    const Run &at = kept[0][wave];
    const bool whole = scalar(at.whole()), first = scalar(at.first()), to_row = row;
    if (!whole && first && tid == 0) P.joins[share] = make_int4(at.s, h, tile, at.sharers());
    uint16_t *op = P.out + row_at * P.ldo + head_at + 8 * half;
    const long long part_at = (2LL * share + (first ? 1 : 0)) * ROWS + wave * 32 + col;
    more = advance(0);
    if (more) open_tile();
    if (rest)
#pragma unroll
      for (int i = 0; i < 2 * NF; ++i) o[i % NF] = mfma32<DT>(vf[i % NF][i / NF], pf[1][i / NF], o[i % NF]);
    float ll = l[0] + l[1];
    ll += __shfl_xor(ll, 32, 64);
    if (whole) {
      const float inv = ll > 0.0f || ll != ll ? 1.0f / ll : 0.0f;                 // (no key seen: zeros)
#pragma unroll
      for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int g = 0; g < 4; g += 2) {         // features 8 g .. 8 g + 15 of the block: the wave's halves have four of each eight, and change them for all of one eight
          uint32_t w[2][2];
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) w[i][j] = pack2<DT>(o[f][4 * (g + i) + 2 * j] * inv, o[f][4 * (g + i) + 2 * j + 1] * inv);
          halves_swap(w[0][0], w[1][0]); halves_swap(w[0][1], w[1][1]);
          if (to_row && ((FULL && KS % 2 == 0) || 32 * f + 8 * (g + half) < D))
            *reinterpret_cast<u32x4_t *>(op + 32 * f + 8 * g) = u32x4_t{w[0][0], w[0][1], w[1][0], w[1][1]};
        }
    } else if (to_row) {
      float *pp = P.part + part_at * C::COLS + 4 * half;
#pragma unroll
      for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int g = 0; g < 4; ++g) *reinterpret_cast<f32x4_t *>(pp + 32 * f + 8 * g) = f32x4_t{o[f][4 * g], o[f][4 * g + 1], o[f][4 * g + 2], o[f][4 * g + 3]};
      if (half == 0) P.part_ml[part_at] = make_float2(ref == NONE ? -__builtin_inff() : -ref, ll);
    }
  } while (more);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // (rows loaded ahead and not used: their place in LDS is this workgroup's until they land)
}

// Joins the partial results of the tiles whose keys several workgroups had (4 to 17 us, the last for 256 tiles of 256 rows with heads of
// 128: up to 67 MB of partial results, just written): workgroup (b, y) takes sixteen rows of the tile that
// begins in share b, whose other parts are the first of the shares after it.  Threads: (group of parts) x (row, 4
// features); the groups' sums are joined in LDS in a fixed order.
template <int DT, int COLS, int ROWS>
__global__ __launch_bounds__(ROWS == 16 ? 1024 : 256) void prompt_join_kernel(const PromptParams P) {
  const int share = blockIdx.x;
  const int4 job = P.joins[share];
  if (job.x < 0) return;
  constexpr int THREADS = ROWS == 16 ? 1024 : 256, QUADS = COLS / 4, SETS = ROWS == 16 ? THREADS / (16 * QUADS) : 1, AHEAD = ROWS == 16 ? 4 : 2;
  static_assert(SETS == 1 || SETS * 16 * QUADS == THREADS, "whole groups");
  __shared__ __attribute__((aligned(16))) float sum_o[SETS > 1 ? SETS * 16 * COLS : 4];
  __shared__ float sum_l[SETS > 1 ? SETS * 16 : 1];
  const PromptSeq seq = prompt_seq(P, job.x);
  const int h = job.y, tile = job.z, parts = job.w, tid = threadIdx.x, r0 = blockIdx.y * 16;
  auto part_at = [&](int i, int r) -> long long { return ((long long)(2 * (share + i)) + (i == 0 ? 1 : 0)) * ROWS + r; };
  for (int x = tid; x < SETS * 16 * QUADS; x += THREADS) {
    const int set = x / (16 * QUADS), item = x - set * 16 * QUADS, rr = item / QUADS, d = (item - rr * QUADS) * 4, r = r0 + rr;
    int token, head;
    const bool row = prompt_row(P, seq, tile, h, r, token, head);
    float mm = -__builtin_inff(), ll = 0.0f;
    f32x4_t y = {0.0f, 0.0f, 0.0f, 0.0f};
    if (row) {
      // (AHEAD loads side by side: the last part stands in for those behind it, and is not added)
      for (int i0 = 0; i0 < parts; i0 += 2 * AHEAD) {
        float t[2 * AHEAD];
#pragma unroll
        for (int i = 0; i < 2 * AHEAD; ++i) t[i] = P.part_ml[part_at(i0 + i < parts ? i0 + i : parts - 1, r)].x;
#pragma unroll
        for (int i = 0; i < 2 * AHEAD; ++i) mm = fmaxf(mm, t[i]);
      }
      for (int i0 = set; i0 < parts; i0 += SETS * AHEAD) {
        float2 ml[AHEAD];
        f32x4_t z[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
          const long long at = part_at(i0 + SETS * i < parts ? i0 + SETS * i : parts - 1, r);
          ml[i] = P.part_ml[at];
          z[i] = *reinterpret_cast<const f32x4_t *>(P.part + at * COLS + d);
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
      *reinterpret_cast<f32x4_t *>(sum_o + (set * 16 + rr) * COLS + d) = y;
      if (d == 0) sum_l[set * 16 + rr] = ll;
      __syncthreads();                                          // (one pass of the loop)
      if (set == 0) {
        ll = 0.0f; y = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < SETS; ++w) {
          ll += sum_l[w * 16 + rr];
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] += sum_o[(w * 16 + rr) * COLS + d + e];
        }
      }
    }
    if (set == 0 && row && d < P.head_dim) {
      const float inv = ll > 0.0f || ll != ll ? 1.0f / ll : 0.0f;
      *reinterpret_cast<uint2 *>(P.out + (long long)(seq.row0 + token) * P.ldo + (long long)head * P.head_dim + d) =
          make_uint2(pack2<DT>(y[0] * inv, y[1] * inv), pack2<DT>(y[2] * inv, y[3] * inv));
    }
  }
}

}  // namespace deinfer
