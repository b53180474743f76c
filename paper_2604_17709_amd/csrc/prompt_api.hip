// Host side of the calls between the projections of a prompt (include/deinfer.h): positions of several axes, norms of
// queries and keys with their rotation, attention over packed keys and values.  Validation on the host only, then one or two
// launches; nothing allocates and nothing synchronises.
#include "../../include/deinfer.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <type_traits>

#include "common.h"
#include "host_common.h"
#include "axis_positions_kernel.h"
#include "norm_rope_kernel.h"
#include "prompt_attention_launch.h"

using namespace deinfer;

namespace {

static_assert(DEINFER_ROPE_MAX_AXES == ROPE_MAX_AXES && DEINFER_NORM_MAX_DIM == NORM_MAX_DIM, "limits of the boundary are those of the kernels");

constexpr int64_t MAX_ROWS = 1 << 28;            // token rows of a call
constexpr int64_t MAX_PITCH = 1 << 26;           // elements from row to row

template <typename TE, int VE, bool WHOLE = true>
void launch_norm_rope(const NormRopeParams &Q, bool inter, hipStream_t s) {
  const dim3 grid((unsigned)(Q.r.T < ROPE_GRID ? Q.r.T : ROPE_GRID), (unsigned)ceil_div(Q.r.T, (int64_t)ROPE_GRID)), block(ROPE_THREADS);
  if (inter) {
    if constexpr (VE >= 2) hipLaunchKernelGGL((norm_rope_store_kernel<TE, VE, true, WHOLE>), grid, block, 0, s, Q);
  } else {
    hipLaunchKernelGGL((norm_rope_store_kernel<TE, VE, false, WHOLE>), grid, block, 0, s, Q);
  }
}

// ---- attention: which kernel, and its workspace
constexpr size_t PROMPT_WS_HEADER = 256;

PromptPlan prompt_plan(int64_t T, int64_t n_seqs, int64_t n_q, int64_t n_kv, int64_t head_dim) {
  PromptPlan p;
  const int64_t per_head = ceil_div(T * (n_q / n_kv), n_seqs > 0 ? n_seqs : 1);      // rows of a sequence and key head, on average
  // Tiles of 16 rows without LDS, of 128 and of 256, in us, heads of 128, 8 key heads.  8 query heads each, 4000 keys: 8 sequences with one
  // token 30.9, 36.8 and 37.5, with two 32.4 and 38.6; 16 with one 49 and (256 rows) 54, 32 107 and 108; 64 with one 201, 191 and 191, with
  // two 205 and 193, with three (two tiles of 16) 390 and 193: up to 16 rows the rule takes the small tiles whatever the sequences' number,
  // which is 5 to 6 % too slow for 64 and more.  One height for all sequences: a chunk of 512 tokens beside 63 single ones, 32 heads
  // each with its own keys, 2000 to 4096 of them, gets 16 rows, 698 us where two calls take 68 and 520.  4 query heads each, whole prompts: 32 of 8 tokens 13.4, 15.1 and 16.3, 32 of 16 15.1, 15.4 and 16.7; from 64 tokens on
  // the last two are equal, and long ones need 256 rows (906 TFLOP/s against 746).
  p.rows = per_head <= 16 ? 16 : head_dim > 128 || per_head <= 128 ? 128 : 256;
  p.cols = p.rows == 16 ? (head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256) : head_dim <= 64 ? 64 : head_dim <= 96 ? 96 : head_dim <= 128 ? 128 : 256;
  const int cus = device_cus();
  p.shares = (p.rows == 16 ? 2 : 1) * (int64_t)(cus > 0 ? cus : 256);
  p.joins = PROMPT_WS_HEADER;
  p.ml = p.joins + (size_t)round_up(2 * (cus > 0 ? cus : 256) * 16, 256);           // (the same for every choice: more rows never need less)
  p.part = p.ml + (size_t)round_up(2 * p.shares * p.rows * 8, 256);
  p.bytes = p.part + (size_t)(2 * p.shares * p.rows * p.cols * 4);
  return p;
}

}  // namespace

extern "C" {

int deinfer_axis_positions(const int32_t *segments, int64_t n_segments, const int32_t *segment_start, const int32_t *row_start,
                           const int32_t *cached, int64_t n_seqs, int64_t T, int32_t *positions, int64_t pitch, void *stream) {
  if (n_segments < 0 || n_seqs < 0 || T < 0 || pitch < 0) return fail(DEINFER_ERR_INVALID_ARG, "axis positions: negative size");
  if (n_seqs > DEINFER_KV_MAX_SEQS || T > MAX_ROWS || n_segments > MAX_ROWS)
    return fail(DEINFER_ERR_UNSUPPORTED, "axis positions: more than %d sequences, 2^28 rows or 2^28 segments", DEINFER_KV_MAX_SEQS);
  if (pitch < T) return fail(DEINFER_ERR_INVALID_ARG, "axis positions: the pitch is smaller than the rows");
  if (T == 0 || n_seqs == 0) return DEINFER_OK;
  if (!segment_start || !row_start || !positions || (n_segments > 0 && !segments)) return fail(DEINFER_ERR_INVALID_ARG, "axis positions: segments, segment_start, row_start or positions is NULL");
  if (!aligned(segments, 16)) return fail(DEINFER_ERR_MISALIGNED, "axis positions: segments must be 16-byte aligned");
  for (const void *p : {(const void *)segment_start, (const void *)row_start, (const void *)cached, (const void *)positions})
    if (!aligned(p, 4)) return fail(DEINFER_ERR_MISALIGNED, "axis positions: a pointer is not 4-byte aligned");
  AxisPositionsParams P;
  P.segments = reinterpret_cast<const int4 *>(segments);
  P.segment_start = segment_start; P.row_start = row_start; P.cached = cached; P.positions = positions;
  P.pitch = pitch; P.n_segments = (int)n_segments; P.n_seqs = (int)n_seqs; P.T = (int)T;
  const int64_t runs = ceil_div(ceil_div(T, n_seqs), (int64_t)PLACE_THREADS);       // of a sequence's rows, on average
  hipLaunchKernelGGL(axis_positions_kernel, dim3((unsigned)(n_seqs < 1024 ? n_seqs : 1024), (unsigned)(runs < 256 ? runs : 256)), dim3(PLACE_THREADS), 0,
                     static_cast<hipStream_t>(stream), P);
  return check_launch("axis positions");
}

int deinfer_rope_axes(int64_t rot_dim, int64_t n_axes, const int32_t *pairs, int turns, uint8_t *axis_of) {
  if (rot_dim <= 0 || rot_dim % 2 != 0 || rot_dim > 2 * ROPE_MAX_PAIRS) return fail(DEINFER_ERR_INVALID_ARG, "rope axes: rot_dim must be even, from 2 to %d", 2 * ROPE_MAX_PAIRS);
  if (n_axes < 1 || n_axes > ROPE_MAX_AXES) return fail(DEINFER_ERR_INVALID_ARG, "rope axes: from 1 to %d axes", ROPE_MAX_AXES);
  if (!pairs || !axis_of) return fail(DEINFER_ERR_INVALID_ARG, "rope axes: pairs or axis_of is NULL");
  int64_t left[ROPE_MAX_AXES], sum = 0;
  for (int64_t a = 0; a < n_axes; ++a) {
    if (pairs[a] < 0) return fail(DEINFER_ERR_INVALID_ARG, "rope axes: a negative number of pairs");
    sum += left[a] = pairs[a];
  }
  if (sum != rot_dim / 2) return fail(DEINFER_ERR_INVALID_ARG, "rope axes: the axes have %lld pairs, rot_dim has %lld", (long long)sum, (long long)(rot_dim / 2));
  for (int64_t i = 0; i < sum;)
    for (int64_t a = 0; a < n_axes; ++a)
      for (int64_t k = turns ? (left[a] > 0) : left[a]; k > 0; --k) { axis_of[i++] = (uint8_t)a; --left[a]; }
  return DEINFER_OK;
}

int deinfer_norm_rope_store(const void *q, int64_t ldq, int64_t n_q_heads, const void *k, int64_t ldk, const void *v, int64_t ldv,
                            int64_t n_kv_heads, int64_t T, int64_t head_dim, int64_t rot_dim, int interleaved,
                            const void *q_weight, const void *k_weight, double eps,
                            const int32_t *positions, int64_t pos_pitch, int64_t n_axes, const uint8_t *axis_of,
                            const double *freqs, double magnitude, const int32_t *slots, int64_t n_slots,
                            void *q_out, int64_t ldqo, void *k_out, int64_t ldko, void *v_out, int64_t ldvo, int dtype, void *stream) {
  if (T < 0 || n_q_heads < 0 || n_kv_heads < 0 || head_dim <= 0 || n_slots < 0) return fail(DEINFER_ERR_INVALID_ARG, "norm rope store: negative size, or head_dim not positive");
  if (dtype != DEINFER_F32 && dtype != DEINFER_BF16 && dtype != DEINFER_F16) return fail(DEINFER_ERR_UNSUPPORTED, "norm rope store: unknown dtype %d", dtype);
  if (rot_dim < 0 || rot_dim % 2 != 0 || rot_dim > head_dim) return fail(DEINFER_ERR_INVALID_ARG, "norm rope store: rot_dim must be even and at most head_dim");
  if (rot_dim > 2 * ROPE_MAX_PAIRS) return fail(DEINFER_ERR_UNSUPPORTED, "norm rope store: rot_dim above %d", 2 * ROPE_MAX_PAIRS);
  if (head_dim > NORM_MAX_DIM) return fail(DEINFER_ERR_UNSUPPORTED, "norm rope store: head_dim above %d", NORM_MAX_DIM);
  if (!std::isfinite(magnitude)) return fail(DEINFER_ERR_INVALID_ARG, "norm rope store: magnitude is not finite");
  if ((q_weight || k_weight) && !(eps >= 0.0 && std::isfinite((float)eps))) return fail(DEINFER_ERR_INVALID_ARG, "norm rope store: eps must not be negative");
  if (T > MAX_ROWS || n_q_heads > MAX_PITCH / head_dim || n_kv_heads > MAX_PITCH / head_dim) return fail(DEINFER_ERR_UNSUPPORTED, "norm rope store: sizes out of range");
  if (n_axes < 1 || n_axes > ROPE_MAX_AXES) return fail(DEINFER_ERR_INVALID_ARG, "norm rope store: from 1 to %d axes", ROPE_MAX_AXES);
  const bool have_q = n_q_heads > 0 && q, have_k = n_kv_heads > 0 && k, have_v = n_kv_heads > 0 && v;
  if (T == 0) return DEINFER_OK;                 // (rows that are none have no address either)
  if ((q == nullptr) != (q_out == nullptr) || (k == nullptr) != (k_out == nullptr) || (v == nullptr) != (v_out == nullptr))
    return fail(DEINFER_ERR_INVALID_ARG, "norm rope store: q, k, v go together with q_out, k_out, v_out");
  if ((q && n_q_heads == 0) || ((k || v) && n_kv_heads == 0)) return fail(DEINFER_ERR_INVALID_ARG, "norm rope store: no heads");
  const int64_t wq = n_q_heads * head_dim, wk = n_kv_heads * head_dim;
  if ((have_q && (ldq < wq || ldqo < wq)) || (have_k && (ldk < wk || ldko < wk)) || (have_v && (ldv < wk || ldvo < wk)))
    return fail(DEINFER_ERR_INVALID_ARG, "norm rope store: a pitch is smaller than heads * head_dim");
  if (!(have_q || have_k || have_v)) return DEINFER_OK;
  const bool turn = rot_dim > 0 && (have_q || have_k);
  if (turn && (!positions || !freqs)) return fail(DEINFER_ERR_INVALID_ARG, "norm rope store: positions or freqs is NULL");
  if (turn && n_axes > 1 && (!axis_of || pos_pitch < T)) return fail(DEINFER_ERR_INVALID_ARG, "norm rope store: several axes need axis_of, and a pitch of positions of T at least");
  if (slots && ((have_k && k == k_out) || (have_v && v == v_out))) return fail(DEINFER_ERR_INVALID_ARG, "norm rope store: keys and values that go to slots cannot stay in place");
  if ((have_q && q == q_out && ldq != ldqo) || (have_k && k == k_out && ldk != ldko) || (have_v && v == v_out && ldv != ldvo))
    return fail(DEINFER_ERR_INVALID_ARG, "norm rope store: in place, both pitches are one");
  const int64_t es = (int64_t)elem_size(dtype);
  const bool inter = interleaved != 0;
  // elements of a load: what divides a head, its rotated part (half of it, where a pair lies half of it apart) and all rows
  int64_t bytes = 16;
  auto fit = [&](uint64_t x) { while (x % (uint64_t)bytes != 0) bytes /= 2; };
  fit((uint64_t)(head_dim * es)); fit((uint64_t)(inter ? rot_dim * es : rot_dim / 2 * es));
  struct { bool have; const void *p; int64_t ld; } rows[8] = {{have_q, q, ldq}, {have_q, q_out, ldqo}, {have_k, k, ldk}, {have_k, k_out, ldko}, {have_v, v, ldv}, {have_v, v_out, ldvo},
                                                             {have_q && q_weight, q_weight, 0}, {have_k && k_weight, k_weight, 0}};
  for (const auto &r : rows) {
    if (!r.have) continue;
    if (!aligned(r.p, (size_t)es)) return fail(DEINFER_ERR_MISALIGNED, "norm rope store: a tensor is not aligned to its element size");
    fit(reinterpret_cast<uintptr_t>(r.p)); fit((uint64_t)(r.ld * es));
  }
  if (!aligned(positions, 4) || !aligned(slots, 4) || !aligned(freqs, 8)) return fail(DEINFER_ERR_MISALIGNED, "norm rope store: positions, slots or freqs is not aligned");
  if (inter && head_dim % 2 != 0) return fail(DEINFER_ERR_UNSUPPORTED, "norm rope store: interleaved pairs need an even head_dim");
  int ve = (int)(bytes / es);
  const bool apart = inter && ve < 2;            // pairs in rows at odd elements: two at a time, each loaded by itself
  if (apart) ve = 2;
  NormRopeParams Q;
  memset(&Q, 0, sizeof(Q));
  RopeStoreParams &P = Q.r;
  P.q = q; P.k = k; P.v = v; P.q_out = q_out; P.k_out = k_out; P.v_out = v_out;
  P.positions = positions; P.slots = slots; P.freqs = freqs;
  P.ldq = ldq; P.ldk = ldk; P.ldv = ldv; P.ldqo = ldqo; P.ldko = ldko; P.ldvo = ldvo; P.n_slots = n_slots;
  P.T = (int)T; P.n_q = have_q ? (int)n_q_heads : 0; P.n_kv = have_k ? (int)n_kv_heads : 0; P.n_v = have_v ? (int)n_kv_heads : 0;
  P.head_dim = (int)head_dim; P.rot_dim = turn ? (int)rot_dim : 0; P.magnitude = (float)magnitude;
  Q.q_weight = have_q ? q_weight : nullptr; Q.k_weight = have_k ? k_weight : nullptr;
  Q.axis_of = n_axes > 1 ? axis_of : nullptr; Q.pos_pitch = pos_pitch; Q.n_axes = (int)n_axes; Q.eps = eps;
  const int pieces = (inter ? P.rot_dim : P.rot_dim / 2) / ve + (P.head_dim - P.rot_dim) / ve;
  Q.lanes = 1;
  while (Q.lanes < pieces && Q.lanes < kWave) Q.lanes *= 2;
  hipStream_t s = static_cast<hipStream_t>(stream);
  by_dtype(dtype, [&](auto tag) {
    using TE = decltype(tag);
    if (apart) launch_norm_rope<TE, 2, false>(Q, true, s);
    else if (sizeof(TE) == 2 && ve == 8) launch_norm_rope<TE, (sizeof(TE) == 2 ? 8 : 4)>(Q, inter, s);
    else if (ve == 4) launch_norm_rope<TE, 4>(Q, inter, s);
    else if (ve == 2) launch_norm_rope<TE, 2>(Q, inter, s);
    else launch_norm_rope<TE, 1>(Q, inter, s);
    return 0;
  });
  return check_launch("norm rope store");
}

int deinfer_prompt_attention_workspace_bytes(int64_t T, int64_t n_seqs, int64_t n_q_heads, int64_t n_kv_heads, int64_t head_dim, size_t *bytes) {
  if (!bytes) return fail(DEINFER_ERR_INVALID_ARG, "bytes is NULL");
  if (T < 0 || n_seqs < 0 || n_q_heads <= 0 || n_kv_heads <= 0 || n_q_heads % n_kv_heads != 0 || head_dim <= 0)
    return fail(DEINFER_ERR_INVALID_ARG, "prompt attention: bad size, or query heads that are no multiple of the key heads");
  if (T > MAX_ROWS || n_q_heads > MAX_PITCH || head_dim > 256) return fail(DEINFER_ERR_UNSUPPORTED, "prompt attention: sizes out of range");
  *bytes = prompt_plan(T, n_seqs, n_q_heads, n_kv_heads, head_dim).bytes;
  return DEINFER_OK;
}

int deinfer_prompt_attention(const void *q, int64_t T, int64_t ldq, int64_t n_q_heads, int64_t n_kv_heads, int64_t head_dim,
                             const int32_t *q_start, const void *k, int64_t ldk, const void *v, int64_t ldv, int64_t n_keys,
                             const int32_t *k_start, int64_t n_seqs, int64_t left, int64_t right, double scale,
                             void *out, int64_t ldo, int dtype, void *ws, size_t ws_bytes, void *stream) {
  if (T < 0 || n_keys < 0 || n_seqs < 0 || n_q_heads <= 0 || n_kv_heads <= 0 || n_q_heads % n_kv_heads != 0)
    return fail(DEINFER_ERR_INVALID_ARG, "prompt attention: bad size, or query heads that are no multiple of the key heads");
  if (dtype != DEINFER_BF16 && dtype != DEINFER_F16) return fail(DEINFER_ERR_UNSUPPORTED, "prompt attention: 16-bit types (bf16, fp16) only");
  if (head_dim <= 0 || head_dim % 8 != 0 || head_dim > 256) return fail(DEINFER_ERR_UNSUPPORTED, "prompt attention: head_dim must be a multiple of 8, from 8 to 256");
  if (!(scale > 0.0) || !std::isfinite(scale)) return fail(DEINFER_ERR_INVALID_ARG, "prompt attention: scale must be positive");
  const float scale2 = (float)(scale * 1.4426950408889634074);      // (0 or infinity times a score would be no number)
  if (!std::isnormal(scale2)) return fail(DEINFER_ERR_UNSUPPORTED, "prompt attention: scale is out of the range of fp32");
  if (T > MAX_ROWS || n_keys > MAX_ROWS || n_seqs > DEINFER_KV_MAX_SEQS || n_q_heads > MAX_PITCH / head_dim)
    return fail(DEINFER_ERR_UNSUPPORTED, "prompt attention: sizes out of range");
  const int64_t wq = n_q_heads * head_dim, wk = n_kv_heads * head_dim;
  if (ldq < wq || ldo < wq || ldk < wk || ldv < wk) return fail(DEINFER_ERR_INVALID_ARG, "prompt attention: a pitch is smaller than heads * head_dim");
  if (ldk > MAX_PITCH || ldv > MAX_PITCH) return fail(DEINFER_ERR_UNSUPPORTED, "prompt attention: a pitch of keys or values above 2^26 elements");
  if (T == 0 || n_seqs == 0) return DEINFER_OK;
  if (!q || !out || !q_start || (n_keys > 0 && (!k || !v))) return fail(DEINFER_ERR_INVALID_ARG, "prompt attention: a pointer is NULL");
  if (out == q || out == k || out == v) return fail(DEINFER_ERR_INVALID_ARG, "prompt attention: out must be a tensor of its own");
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || ldq % 8 || ldk % 8 || ldv % 8 || ldo % 8)
    return fail(DEINFER_ERR_MISALIGNED, "prompt attention: q, k, v and out must be 16-byte aligned, their pitches multiples of 8");
  if (!aligned(q_start, 4) || !aligned(k_start, 4)) return fail(DEINFER_ERR_MISALIGNED, "prompt attention: a list is not 4-byte aligned");
  const PromptPlan pl = prompt_plan(T, n_seqs, n_q_heads, n_kv_heads, head_dim);
  if (!ws || ws_bytes < pl.bytes) return fail(DEINFER_ERR_WORKSPACE, "prompt attention: workspace of %zu bytes, %zu needed", ws ? ws_bytes : (size_t)0, pl.bytes);
  if (!aligned(ws, 256)) return fail(DEINFER_ERR_MISALIGNED, "prompt attention: the workspace must be 256-byte aligned");
  PromptParams P;
  memset(&P, 0, sizeof(P));
  P.q = static_cast<const uint16_t *>(q); P.k = static_cast<const uint16_t *>(k); P.v = static_cast<const uint16_t *>(v);
  P.out = static_cast<uint16_t *>(out);
  P.q_start = q_start; P.k_start = k_start;
  P.ldq = ldq; P.ldo = ldo; P.ldk = (uint32_t)(2 * ldk); P.ldv = (uint32_t)(2 * ldv);
  P.T = (int)T; P.Tk = (int)n_keys; P.n_seqs = (int)n_seqs; P.head_dim = (int)head_dim; P.group = (int)(n_q_heads / n_kv_heads);
  P.head_tiles = (int)ceil_div(P.group, pl.rows); P.tile_group = (int)ceil_div(P.group, P.head_tiles); P.tile_tokens = pl.rows / P.tile_group;
  P.heads = (int)n_kv_heads * P.head_tiles; P.per_token = 1.0 / P.tile_tokens;
  P.per_workgroup = 1.0 / (double)pl.shares;
  P.left = left < 0 || left > PROMPT_FAR ? PROMPT_FAR : (int)left;
  P.right = right < 0 || right > PROMPT_FAR ? PROMPT_FAR : (int)right;
  P.scale2 = scale2;
  P.n_shares = (int)pl.shares;
  char *w = static_cast<char *>(ws);
  P.joins = reinterpret_cast<int4 *>(w + pl.joins);
  P.part_ml = reinterpret_cast<float2 *>(w + pl.ml);
  P.part = reinterpret_cast<float *>(w + pl.part);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return dtype == DEINFER_F16 ? launch_prompt_f16(pl, P, s) : launch_prompt_bf16(pl, P, s);
}

}  // extern "C"
