// Host side of the calls around a paged cache (include/deinfer.h): from the requests' lengths to the
// attention that reads the cache.  Validation on the host only, then one or two launches; nothing allocates
// and nothing synchronises.
#include "../../include/deinfer.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <type_traits>

#include "common.h"
#include "host_common.h"
#include "step_kernels.h"
#include "rope_store_kernel.h"
#include "tree_attention_kernel.h"

using namespace deinfer;

namespace {

static_assert(DEINFER_KV_MAX_SEQS == STEP_MAX_SEQS && DEINFER_TREE_MAX_WORDS == TREE_MAX_WORDS, "limits of the boundary are those of the kernels");
static_assert(DEINFER_KV_PLAN_BAD_BLOCK == KV_PLAN_BAD_BLOCK && DEINFER_KV_PLAN_BUFFER_FULL == KV_PLAN_BUFFER_FULL &&
              DEINFER_KV_PLAN_TABLE_FULL == KV_PLAN_TABLE_FULL && DEINFER_KV_PLAN_RUNS_FULL == KV_PLAN_RUNS_FULL, "flags of the plan");

constexpr int64_t MAX_ROWS = 1 << 28;            // token rows of a call
constexpr int64_t MAX_PITCH = 1 << 26;           // elements from row to row

int check_pages(const char *what, int64_t n_seqs, int64_t table_pitch, int64_t n_pool_blocks, int64_t block_tokens) {
  if (n_seqs < 0 || table_pitch < 0 || n_pool_blocks < 0 || block_tokens <= 0)
    return fail(DEINFER_ERR_INVALID_ARG, "%s: negative size, or block_tokens not positive", what);
  if (n_seqs > DEINFER_KV_MAX_SEQS) return fail(DEINFER_ERR_UNSUPPORTED, "%s: more than %d sequences", what, DEINFER_KV_MAX_SEQS);
  if (block_tokens > INT32_MAX || n_pool_blocks > INT32_MAX / block_tokens || table_pitch > INT32_MAX / block_tokens)
    return fail(DEINFER_ERR_INVALID_ARG, "%s: more than 2^31 - 1 token slots in the pool or in a row of the block table", what);
  return DEINFER_OK;
}

// ---- attention: which kernel, and its workspace
struct AttPlan {
  int dp, rows;                                  // padded head dimension, rows of a tile
  int64_t shares;
  size_t joins, ml, part, bytes;                 // offsets into the workspace, and its size
};
constexpr size_t ATT_WS_HEADER = 256;

AttPlan att_plan(int64_t T, int64_t n_seqs, int64_t n_q, int64_t n_kv, int64_t head_dim) {
  AttPlan p;
  p.dp = head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256;
  const int64_t per_head = ceil_div(T * (n_q / n_kv), n_seqs > 0 ? n_seqs : 1);      // rows of a sequence and key head, on average
  // Rows of a tile, by the rows there are.  Keys straight into registers for up to 16 rows (8 x 1000 cached tokens, 8 key heads
  // of 128: 18.4 us against 21.1 with tiles of 128; 8 x 4000: 37.5 and 37.3; with 24 rows 54 and 37.6), tiles of 128 up to as many
  // (8 x 4000 with 128 rows: 52 against 54 with 256; 32 x 4000: 122 and 120; 160 rows: 224 and 157).  The sums of 256 rows of 256
  // features have no room in the registers.  One choice for all sequences, from the rows that the buffer has: 255 single tokens
  // on up to 4000 and a chunk of 2048 on 2000 take 588 us in 16-row tiles where the two parts alone take 433 + 77 (8 query and
  // key heads of 128; with 64 query heads 827 and 442 + 284), the single tokens in a buffer with 8192 rows 420 (467 against 442).
  p.rows = per_head <= 16 ? 16 : p.dp == 256 || per_head <= 128 ? 128 : 256;
  const int cus = device_cus();
  p.shares = (p.rows == 16 ? 2 : 1) * (int64_t)(cus > 0 ? cus : 256);
  p.joins = ATT_WS_HEADER;
  p.ml = p.joins + (size_t)round_up(p.shares * 16, 256);
  p.part = p.ml + (size_t)round_up(2 * p.shares * p.rows * 8, 256);
  p.bytes = p.part + (size_t)(2 * p.shares * p.rows * p.dp * 4);
  return p;
}

template <int DT, int DP, bool FULL, bool POW2, int RT>
int launch_attention_tiles(const AttPlan &pl, const AttParams &P, hipStream_t s) {
  using C = AttTile<DP>;
  if (C::LDS > 64 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void *>(&tree_attention_tile_kernel<DT, DP, FULL, POW2, RT>),
                                                hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS) != hipSuccess)
    return fail(DEINFER_ERR_DEVICE, "tree attention: LDS size refused");
  hipLaunchKernelGGL((tree_attention_tile_kernel<DT, DP, FULL, POW2, RT>), dim3((unsigned)pl.shares), dim3(C::THREADS), C::LDS, s, P);
  if (int rc = check_launch("tree attention")) return rc;
  hipLaunchKernelGGL((tree_attention_join_kernel<DT, DP, 128 * RT>), dim3((unsigned)pl.shares, 8 * RT), dim3(JOIN_THREADS<128 * RT>), 0, s, P);
  return check_launch("tree attention");
}
template <int DT, int DP, bool FULL, bool POW2>
int launch_attention(const AttPlan &pl, const AttParams &P, hipStream_t s) {
  if (pl.rows == 128) return launch_attention_tiles<DT, DP, FULL, POW2, 1>(pl, P, s);
  if constexpr (DP < 256)
    if (pl.rows == 256) return launch_attention_tiles<DT, DP, FULL, POW2, 2>(pl, P, s);
  hipLaunchKernelGGL((tree_attention_kernel<DT, DP, FULL, POW2>), dim3((unsigned)pl.shares), dim3(ATT_THREADS), 0, s, P);
  if (int rc = check_launch("tree attention")) return rc;
  hipLaunchKernelGGL((tree_attention_join_kernel<DT, DP, 16>), dim3((unsigned)pl.shares), dim3(JOIN_THREADS<16>), 0, s, P);
  return check_launch("tree attention");
}
template <int DT, int DP>
int launch_attention_of(const AttPlan &pl, const AttParams &P, hipStream_t s) {
  if (P.block_shift < 4) return launch_attention<DT, DP, false, false>(pl, P, s);
  if (P.head_dim == DP) return launch_attention<DT, DP, true, true>(pl, P, s);
  return launch_attention<DT, DP, false, true>(pl, P, s);
}

template <typename TE>
void launch_rope_store(const RopeStoreParams &P, bool vec, bool inter, hipStream_t s) {
  const dim3 grid((unsigned)(P.T < ROPE_GRID ? P.T : ROPE_GRID), (unsigned)ceil_div(P.T, (int64_t)ROPE_GRID)), block(ROPE_THREADS);
  if (vec && inter) hipLaunchKernelGGL((rope_store_kernel<TE, 16 / sizeof(TE), true>), grid, block, 0, s, P);
  else if (vec) hipLaunchKernelGGL((rope_store_kernel<TE, 16 / sizeof(TE), false>), grid, block, 0, s, P);
  else if (inter) hipLaunchKernelGGL((rope_store_kernel<TE, 2, true>), grid, block, 0, s, P);
  else hipLaunchKernelGGL((rope_store_kernel<TE, 1, false>), grid, block, 0, s, P);
}

}  // namespace

extern "C" {

int deinfer_kv_step(const int32_t *cached, const int32_t *n_new, int64_t n_seqs, const int32_t *free_list, int64_t n_free,
                    const int32_t *free_first, int64_t n_pool_blocks, int64_t block_tokens, int32_t *block_table,
                    int64_t table_pitch, int64_t T, int32_t *row_start, int32_t *slots, int32_t *positions, int32_t *counts,
                    void *stream) {
  if (int rc = check_pages("kv step", n_seqs, table_pitch, n_pool_blocks, block_tokens)) return rc;
  if (T < 0 || n_free < 0) return fail(DEINFER_ERR_INVALID_ARG, "kv step: negative size");
  if (T > MAX_ROWS || n_free > INT32_MAX / 2) return fail(DEINFER_ERR_UNSUPPORTED, "kv step: more than 2^28 rows or 2^30 free blocks");
  if (T == 0 && !row_start && !counts) return DEINFER_OK;
  if (!row_start || !counts || (T > 0 && (!slots || !positions))) return fail(DEINFER_ERR_INVALID_ARG, "kv step: an output is NULL");
  if (n_seqs > 0 && (!cached || !n_new || (table_pitch > 0 && !block_table))) return fail(DEINFER_ERR_INVALID_ARG, "kv step: lengths or block table are NULL");
  if (n_free > 0 && !free_list) return fail(DEINFER_ERR_INVALID_ARG, "kv step: free_list is NULL");
  if (free_first && free_first >= counts && free_first < counts + 4) return fail(DEINFER_ERR_INVALID_ARG, "kv step: free_first must not lie in counts");
  for (const void *p : {(const void *)cached, (const void *)n_new, (const void *)free_list, (const void *)free_first,
                        (const void *)block_table, (const void *)row_start, (const void *)slots, (const void *)positions, (const void *)counts})
    if (!aligned(p, 4)) return fail(DEINFER_ERR_MISALIGNED, "kv step: a pointer is not 4-byte aligned");
  KvStepParams P;
  P.cached = cached; P.n_new = n_new; P.free_list = free_list; P.free_first = free_first;
  P.table = block_table; P.row_start = row_start; P.slots = slots; P.positions = positions; P.counts = counts;
  P.table_pitch = table_pitch; P.n_free = n_free; P.n_pool_blocks = n_pool_blocks;
  P.n_seqs = (int)n_seqs; P.block_tokens = (int)block_tokens; P.T = (int)T;
  P.vec = aligned(slots, 16) && aligned(positions, 16);
  const int64_t groups = T > 0 ? ceil_div(T, (int64_t)STEP_THREADS * STEP_ROWS) : 1;
  hipLaunchKernelGGL(kv_step_kernel, dim3((unsigned)(groups < 512 ? groups : 512)), dim3(STEP_THREADS), 0, static_cast<hipStream_t>(stream), P);
  return check_launch("kv step");
}

int deinfer_kv_compact_plan_device(const int32_t *block_table, int64_t n_seqs, int64_t table_pitch, const int32_t *n_tokens,
                                   const int32_t *n_new, int64_t n_pool_blocks, int64_t buffer_blocks, int64_t block_tokens,
                                   int32_t *plan, int64_t plan_capacity_runs, int32_t *remap, int64_t remap_pitch,
                                   int32_t *positions, void *stream) {
  if (int rc = check_pages("kv plan", n_seqs, table_pitch, n_pool_blocks, block_tokens)) return rc;
  if (buffer_blocks < 0 || plan_capacity_runs < 0 || remap_pitch < 0) return fail(DEINFER_ERR_INVALID_ARG, "kv plan: negative size");
  if (buffer_blocks > INT32_MAX / 2 / block_tokens || plan_capacity_runs > (INT32_MAX - KV_PLAN_HEADER) / 3 || remap_pitch > INT32_MAX)
    return fail(DEINFER_ERR_INVALID_ARG, "kv plan: more than 2^30 token slots in the buffer, or too many runs");
  if (!plan) return fail(DEINFER_ERR_INVALID_ARG, "kv plan: plan is NULL");
  if (n_seqs > 0 && (!n_tokens || (table_pitch > 0 && !block_table))) return fail(DEINFER_ERR_INVALID_ARG, "kv plan: block table or lengths are NULL");
  for (const void *p : {(const void *)block_table, (const void *)n_tokens, (const void *)n_new, (const void *)plan, (const void *)remap, (const void *)positions})
    if (!aligned(p, 4)) return fail(DEINFER_ERR_MISALIGNED, "kv plan: a pointer is not 4-byte aligned");
  KvPlanParams P;
  P.table = block_table; P.n_tokens = n_tokens; P.n_new = n_new; P.plan = plan; P.remap = remap; P.positions = positions;
  P.table_pitch = table_pitch; P.remap_pitch = remap_pitch; P.n_pool_blocks = n_pool_blocks; P.buffer_blocks = buffer_blocks;
  P.capacity = plan_capacity_runs; P.n_seqs = (int)n_seqs; P.block_tokens = (int)block_tokens;
  P.n_chunks = (int)(buffer_blocks > 0 ? ceil_div(buffer_blocks, (int64_t)PLAN_CHUNK) : 1);
  const int64_t items = (remap ? n_seqs * remap_pitch : 0) > (positions ? buffer_blocks : 0) ? n_seqs * remap_pitch : positions ? buffer_blocks : 0;
  const int64_t fill = ceil_div(items, (int64_t)STEP_THREADS);
  hipLaunchKernelGGL(kv_plan_kernel, dim3((unsigned)(P.n_chunks + (fill < 256 ? fill : 256))), dim3(STEP_THREADS), 0, static_cast<hipStream_t>(stream), P);
  return check_launch("kv plan");
}

int deinfer_tree_mask(const int32_t *parents, const int32_t *row_start, const int32_t *cached, int64_t n_seqs, int64_t T,
                      uint32_t *mask, int64_t mask_words, int32_t *positions, void *stream) {
  if (n_seqs < 0 || T < 0 || mask_words <= 0) return fail(DEINFER_ERR_INVALID_ARG, "tree mask: negative size, or mask_words not positive");
  if (mask_words > DEINFER_TREE_MAX_WORDS) return fail(DEINFER_ERR_UNSUPPORTED, "tree mask: more than %d words (%d drafted tokens) per row", DEINFER_TREE_MAX_WORDS, 32 * DEINFER_TREE_MAX_WORDS);
  if (n_seqs > DEINFER_KV_MAX_SEQS || T > MAX_ROWS) return fail(DEINFER_ERR_UNSUPPORTED, "tree mask: more than %d sequences or 2^28 rows", DEINFER_KV_MAX_SEQS);
  if (T == 0 || n_seqs == 0) return DEINFER_OK;
  if (!parents || !row_start || !cached || !mask) return fail(DEINFER_ERR_INVALID_ARG, "tree mask: parents, row_start, cached or mask is NULL");
  for (const void *p : {(const void *)parents, (const void *)row_start, (const void *)cached, (const void *)mask, (const void *)positions})
    if (!aligned(p, 4)) return fail(DEINFER_ERR_MISALIGNED, "tree mask: a pointer is not 4-byte aligned");
  const int lds = tree_mask_lds((int)mask_words);
  if (lds > 64 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void *>(&tree_mask_kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                             tree_mask_lds(TREE_MAX_WORDS)) != hipSuccess)
    return fail(DEINFER_ERR_DEVICE, "tree mask: LDS size refused");
  hipLaunchKernelGGL(tree_mask_kernel, dim3((unsigned)(n_seqs < 1024 ? n_seqs : 1024)), dim3(mask_words == 1 ? 256 : TREE_THREADS), (size_t)lds, static_cast<hipStream_t>(stream),
                     parents, row_start, cached, (int)n_seqs, (int)T, mask, (int)mask_words, positions);
  return check_launch("tree mask");
}

int deinfer_rope_frequencies(int64_t rot_dim, double theta, const deinfer_rope_scaling_t *scaling, double *freqs, double *magnitude) {
  if (rot_dim <= 0 || rot_dim % 2 != 0 || rot_dim > 2 * ROPE_MAX_PAIRS) return fail(DEINFER_ERR_INVALID_ARG, "rope frequencies: rot_dim must be even, from 2 to %d", 2 * ROPE_MAX_PAIRS);
  if (!(theta > 0.0) || !std::isfinite(theta)) return fail(DEINFER_ERR_INVALID_ARG, "rope frequencies: theta must be positive");
  if (!freqs) return fail(DEINFER_ERR_INVALID_ARG, "rope frequencies: freqs is NULL");
  deinfer_rope_scaling_t sc;
  memset(&sc, 0, sizeof(sc));
  if (scaling) sc = *scaling;
  const double two_pi = 6.283185307179586476925;
  if (sc.kind != DEINFER_ROPE_PLAIN && !(sc.factor > 0.0 && std::isfinite(sc.factor))) return fail(DEINFER_ERR_INVALID_ARG, "rope frequencies: factor must be positive");
  if (sc.kind == DEINFER_ROPE_BANDS || sc.kind == DEINFER_ROPE_RAMP) {
    if (!(sc.original_context > 0.0) || !(sc.low > 0.0) || !(sc.high > sc.low) || !std::isfinite(sc.high) || !std::isfinite(sc.original_context))
      return fail(DEINFER_ERR_INVALID_ARG, "rope frequencies: original_context > 0 and 0 < low < high are required");
  }
  if (sc.kind == DEINFER_ROPE_RAMP && !(theta > 1.0)) return fail(DEINFER_ERR_INVALID_ARG, "rope frequencies: the ramp needs theta > 1");
  const double D = (double)rot_dim;
  double base = theta;
  switch (sc.kind) {
    case DEINFER_ROPE_PLAIN: case DEINFER_ROPE_LINEAR: case DEINFER_ROPE_BANDS: case DEINFER_ROPE_RAMP: break;
    case DEINFER_ROPE_BASE:
      if (rot_dim <= 2) return fail(DEINFER_ERR_INVALID_ARG, "rope frequencies: a change of base needs rot_dim > 2");
      base = theta * std::pow(sc.factor, D / (D - 2.0));
      break;
    default: return fail(DEINFER_ERR_UNSUPPORTED, "rope frequencies: unknown kind %d", sc.kind);
  }
  // ramp: the pair that turns `t` times within the original context, as a real number
  auto pair_of_turns = [&](double t) { return D * std::log(sc.original_context / (two_pi * t)) / (2.0 * std::log(theta)); };
  double from = 0.0, to = 1.0;
  if (sc.kind == DEINFER_ROPE_RAMP) {
    from = std::floor(pair_of_turns(sc.high)); to = std::ceil(pair_of_turns(sc.low));
    from = from < 0.0 ? 0.0 : from; to = to > D - 1.0 ? D - 1.0 : to;
    if (to <= from) to = from + 0.001;
  }
  for (int64_t i = 0; i < rot_dim / 2; ++i) {
    const double f = std::pow(base, -2.0 * (double)i / D);
    double keep = 1.0;                           // share of the unscaled frequency
    if (sc.kind == DEINFER_ROPE_LINEAR) keep = 0.0;
    if (sc.kind == DEINFER_ROPE_BANDS) keep = (sc.original_context * f / two_pi - sc.low) / (sc.high - sc.low);
    if (sc.kind == DEINFER_ROPE_RAMP) keep = 1.0 - ((double)i - from) / (to - from);
    keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
    freqs[i] = sc.kind == DEINFER_ROPE_PLAIN || sc.kind == DEINFER_ROPE_BASE ? f : keep * f + (1.0 - keep) * f / sc.factor;
  }
  if (magnitude) *magnitude = sc.kind == DEINFER_ROPE_RAMP && sc.factor > 1.0 ? 0.1 * std::log(sc.factor) + 1.0 : 1.0;
  return DEINFER_OK;
}

int deinfer_rope_store(const void *q, int64_t ldq, int64_t n_q_heads, const void *k, int64_t ldk, const void *v, int64_t ldv,
                       int64_t n_kv_heads, int64_t T, int64_t head_dim, int64_t rot_dim, int interleaved,
                       const int32_t *positions, const double *freqs, double magnitude, const int32_t *slots, int64_t n_slots,
                       void *q_out, int64_t ldqo, void *k_out, int64_t ldko, void *v_out, int64_t ldvo, int dtype, void *stream) {
  if (T < 0 || n_q_heads < 0 || n_kv_heads < 0 || head_dim <= 0 || n_slots < 0) return fail(DEINFER_ERR_INVALID_ARG, "rope store: negative size, or head_dim not positive");
  if (dtype != DEINFER_F32 && dtype != DEINFER_BF16 && dtype != DEINFER_F16) return fail(DEINFER_ERR_UNSUPPORTED, "rope store: unknown dtype %d", dtype);
  if (rot_dim < 0 || rot_dim % 2 != 0 || rot_dim > head_dim) return fail(DEINFER_ERR_INVALID_ARG, "rope store: rot_dim must be even and at most head_dim");
  if (rot_dim > 2 * ROPE_MAX_PAIRS) return fail(DEINFER_ERR_UNSUPPORTED, "rope store: rot_dim above %d", 2 * ROPE_MAX_PAIRS);
  if (!std::isfinite(magnitude)) return fail(DEINFER_ERR_INVALID_ARG, "rope store: magnitude is not finite");
  if (T > MAX_ROWS || head_dim > MAX_PITCH || n_q_heads > MAX_PITCH / head_dim || n_kv_heads > MAX_PITCH / head_dim)
    return fail(DEINFER_ERR_UNSUPPORTED, "rope store: sizes out of range");
  const bool have_q = n_q_heads > 0 && q, have_k = n_kv_heads > 0 && k, have_v = n_kv_heads > 0 && v;
  if (T == 0) return DEINFER_OK;                 // (rows that are none have no address either)
  if ((q == nullptr) != (q_out == nullptr) || (k == nullptr) != (k_out == nullptr) || (v == nullptr) != (v_out == nullptr))
    return fail(DEINFER_ERR_INVALID_ARG, "rope store: q, k, v go together with q_out, k_out, v_out");
  if ((q && n_q_heads == 0) || ((k || v) && n_kv_heads == 0)) return fail(DEINFER_ERR_INVALID_ARG, "rope store: no heads");
  const int64_t wq = n_q_heads * head_dim, wk = n_kv_heads * head_dim;
  if ((have_q && (ldq < wq || ldqo < wq)) || (have_k && (ldk < wk || ldko < wk)) || (have_v && (ldv < wk || ldvo < wk)))
    return fail(DEINFER_ERR_INVALID_ARG, "rope store: a pitch is smaller than heads * head_dim");
  if (!(have_q || have_k || have_v)) return DEINFER_OK;
  if (rot_dim > 0 && (have_q || have_k) && (!positions || !freqs)) return fail(DEINFER_ERR_INVALID_ARG, "rope store: positions or freqs is NULL");
  if (slots && ((have_k && k == k_out) || (have_v && v == v_out))) return fail(DEINFER_ERR_INVALID_ARG, "rope store: keys and values that go to slots cannot stay in place");
  if ((have_q && q == q_out && ldq != ldqo) || (have_k && k == k_out && ldk != ldko) || (have_v && v == v_out && ldv != ldvo))
    return fail(DEINFER_ERR_INVALID_ARG, "rope store: in place, both pitches are one");
  const size_t es = elem_size(dtype);
  bool vec = head_dim * es % 16 == 0 && rot_dim * es % (interleaved ? 16 : 32) == 0;
  struct { bool have; const void *p; int64_t ld; } rows[6] = {{have_q, q, ldq}, {have_q, q_out, ldqo}, {have_k, k, ldk}, {have_k, k_out, ldko}, {have_v, v, ldv}, {have_v, v_out, ldvo}};
  for (const auto &r : rows) {
    if (!r.have) continue;
    if (!aligned(r.p, es)) return fail(DEINFER_ERR_MISALIGNED, "rope store: a tensor is not aligned to its element size");
    vec = vec && aligned(r.p, 16) && r.ld * es % 16 == 0;
  }
  if (!aligned(positions, 4) || !aligned(slots, 4) || !aligned(freqs, 8)) return fail(DEINFER_ERR_MISALIGNED, "rope store: positions, slots or freqs is not aligned");
  if (!vec && interleaved && head_dim % 2 != 0) return fail(DEINFER_ERR_UNSUPPORTED, "rope store: interleaved pairs need an even head_dim");
  RopeStoreParams P;
  memset(&P, 0, sizeof(P));
  P.q = q; P.k = k; P.v = v; P.q_out = q_out; P.k_out = k_out; P.v_out = v_out;
  P.positions = positions; P.slots = slots; P.freqs = freqs;
  P.ldq = ldq; P.ldk = ldk; P.ldv = ldv; P.ldqo = ldqo; P.ldko = ldko; P.ldvo = ldvo; P.n_slots = n_slots;
  P.T = (int)T; P.n_q = have_q ? (int)n_q_heads : 0; P.n_kv = have_k ? (int)n_kv_heads : 0; P.n_v = have_v ? (int)n_kv_heads : 0;
  P.head_dim = (int)head_dim; P.rot_dim = have_q || have_k ? (int)rot_dim : 0; P.magnitude = (float)magnitude;
  by_dtype(dtype, [&](auto tag) {
    launch_rope_store<decltype(tag)>(P, vec, interleaved != 0, static_cast<hipStream_t>(stream));
    return 0;
  });
  return check_launch("rope store");
}

int deinfer_tree_attention_workspace_bytes(int64_t T, int64_t n_seqs, int64_t n_q_heads, int64_t n_kv_heads, int64_t head_dim, size_t *bytes) {
  if (!bytes) return fail(DEINFER_ERR_INVALID_ARG, "bytes is NULL");
  if (T < 0 || n_seqs < 0 || n_q_heads <= 0 || n_kv_heads <= 0 || n_q_heads % n_kv_heads != 0 || head_dim <= 0)
    return fail(DEINFER_ERR_INVALID_ARG, "tree attention: bad size, or query heads that are no multiple of the key heads");
  if (T > MAX_ROWS || n_q_heads > MAX_PITCH || T * n_q_heads > INT32_MAX / 2 || head_dim > 256) return fail(DEINFER_ERR_UNSUPPORTED, "tree attention: sizes out of range");
  *bytes = att_plan(T, n_seqs, n_q_heads, n_kv_heads, head_dim).bytes;
  return DEINFER_OK;
}

int deinfer_tree_attention(const void *q, int64_t T, int64_t ldq, int64_t n_q_heads, int64_t n_kv_heads, int64_t head_dim,
                           const int32_t *row_start, const int32_t *cached, int64_t n_seqs, const uint32_t *mask, int64_t mask_words,
                           const void *k_pool, int64_t ldk, const void *v_pool, int64_t ldv, int64_t n_pool_blocks, int64_t block_tokens,
                           const int32_t *block_table, int64_t table_pitch, double scale, void *out, int64_t ldo, int dtype,
                           void *ws, size_t ws_bytes, void *stream) {
  if (int rc = check_pages("tree attention", n_seqs, table_pitch, n_pool_blocks, block_tokens)) return rc;
  if (T < 0 || n_q_heads <= 0 || n_kv_heads <= 0 || n_q_heads % n_kv_heads != 0)
    return fail(DEINFER_ERR_INVALID_ARG, "tree attention: bad size, or query heads that are no multiple of the key heads");
  if (dtype != DEINFER_BF16 && dtype != DEINFER_F16) return fail(DEINFER_ERR_UNSUPPORTED, "tree attention: 16-bit types (bf16, fp16) only");
  if (head_dim <= 0 || head_dim % 8 != 0 || head_dim > 256) return fail(DEINFER_ERR_UNSUPPORTED, "tree attention: head_dim must be a multiple of 8, from 8 to 256");
  if (!(scale > 0.0) || !std::isfinite(scale)) return fail(DEINFER_ERR_INVALID_ARG, "tree attention: scale must be positive");
  const float scale2 = (float)(scale * 1.4426950408889634074);      // (0 or infinity times a score would be no number)
  if (!std::isnormal(scale2)) return fail(DEINFER_ERR_UNSUPPORTED, "tree attention: scale is out of the range of fp32");
  if (T > MAX_ROWS || n_q_heads > MAX_PITCH / head_dim || T * n_q_heads > INT32_MAX / 2) return fail(DEINFER_ERR_UNSUPPORTED, "tree attention: sizes out of range");
  if (mask && (mask_words <= 0 || mask_words > DEINFER_TREE_MAX_WORDS)) return fail(DEINFER_ERR_INVALID_ARG, "tree attention: mask_words must be from 1 to %d", DEINFER_TREE_MAX_WORDS);
  const int64_t wq = n_q_heads * head_dim, wk = n_kv_heads * head_dim;
  if (ldq < wq || ldo < wq || ldk < wk || ldv < wk) return fail(DEINFER_ERR_INVALID_ARG, "tree attention: a pitch is smaller than heads * head_dim");
  if (ldk > MAX_PITCH || ldv > MAX_PITCH) return fail(DEINFER_ERR_UNSUPPORTED, "tree attention: a pitch of the cache above 2^26 elements");
  if (T == 0 || n_seqs == 0) return DEINFER_OK;
  if (table_pitch * block_tokens > INT32_MAX / 2) return fail(DEINFER_ERR_UNSUPPORTED, "tree attention: more than 2^30 tokens in a row of the block table");
  if (n_pool_blocks == 0 || table_pitch == 0) return fail(DEINFER_ERR_INVALID_ARG, "tree attention: an empty pool or block table");
  if (!q || !k_pool || !v_pool || !out || !row_start || !cached || !block_table) return fail(DEINFER_ERR_INVALID_ARG, "tree attention: a pointer is NULL");
  if (out == q) return fail(DEINFER_ERR_INVALID_ARG, "tree attention: out must not be q");
  if (!aligned(q, 16) || !aligned(k_pool, 16) || !aligned(v_pool, 16) || !aligned(out, 16) || ldq % 8 || ldk % 8 || ldv % 8 || ldo % 8)
    return fail(DEINFER_ERR_MISALIGNED, "tree attention: q, the pools and out must be 16-byte aligned, their pitches multiples of 8");
  if (!aligned(row_start, 4) || !aligned(cached, 4) || !aligned(block_table, 4) || !aligned(mask, 4)) return fail(DEINFER_ERR_MISALIGNED, "tree attention: a list is not 4-byte aligned");
  const AttPlan pl = att_plan(T, n_seqs, n_q_heads, n_kv_heads, head_dim);
  if (!ws || ws_bytes < pl.bytes) return fail(DEINFER_ERR_WORKSPACE, "tree attention: workspace of %zu bytes, %zu needed", ws ? ws_bytes : (size_t)0, pl.bytes);
  if (!aligned(ws, 256)) return fail(DEINFER_ERR_MISALIGNED, "tree attention: the workspace must be 256-byte aligned");
  AttParams P;
  memset(&P, 0, sizeof(P));
  P.q = static_cast<const uint16_t *>(q); P.k = static_cast<const uint16_t *>(k_pool); P.v = static_cast<const uint16_t *>(v_pool);
  P.out = static_cast<uint16_t *>(out);
  P.row_start = row_start; P.cached = cached; P.table = block_table; P.mask = mask;
  P.ldq = ldq; P.ldk = (uint32_t)(2 * ldk); P.ldv = (uint32_t)(2 * ldv); P.ldo = ldo; P.table_pitch = (int)table_pitch; P.n_pool_blocks = (int)n_pool_blocks;
  P.most_keys = (int)(table_pitch * block_tokens);
  P.T = (int)T; P.n_seqs = (int)n_seqs; P.n_kv = (int)n_kv_heads; P.group = (int)(n_q_heads / n_kv_heads); P.head_dim = (int)head_dim;
  P.block_tokens = (int)block_tokens; P.mask_words = (int)mask_words;
  P.block_shift = 0;
  if ((block_tokens & (block_tokens - 1)) == 0) while ((1LL << P.block_shift) < block_tokens) ++P.block_shift;
  P.scale2 = scale2;
  P.n_shares = (int)pl.shares;
  char *w = static_cast<char *>(ws);
  P.joins = reinterpret_cast<int4 *>(w + pl.joins);
  P.part_ml = reinterpret_cast<float2 *>(w + pl.ml);
  P.part = reinterpret_cast<float *>(w + pl.part);
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto by_dim = [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    if (pl.dp == 64) return launch_attention_of<DT, 64>(pl, P, s);
    if (pl.dp == 128) return launch_attention_of<DT, 128>(pl, P, s);
    return launch_attention_of<DT, 256>(pl, P, s);
  };
  if (dtype == DEINFER_F16) return by_dim(std::integral_constant<int, DT_F16>{});
  return by_dim(std::integral_constant<int, DT_BF16>{});
}

}  // extern "C"
