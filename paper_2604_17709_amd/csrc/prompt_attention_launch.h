// Launches of the attention over packed keys and values; one source for each storage type instantiates them.
#pragma once
#include "host_common.h"
#include "prompt_attention_kernel.h"

namespace deinfer {

struct PromptPlan {
  int rows, cols;                                // of a tile
  int64_t shares;
  size_t joins, ml, part, bytes;                 // offsets into the workspace, and its size
};

DEINFER_HIDDEN int launch_prompt_bf16(const PromptPlan &pl, const PromptParams &P, hipStream_t s);
DEINFER_HIDDEN int launch_prompt_f16(const PromptPlan &pl, const PromptParams &P, hipStream_t s);

template <int DT, int KS, int WAVES, bool FULL>
int launch_prompt_tiles(const PromptPlan &pl, const PromptParams &P, hipStream_t s) {
  using C = PromptTile<KS, WAVES>;
  if (C::LDS > 64 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void *>(&prompt_tile_kernel<DT, KS, WAVES, FULL>),
                                                hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS) != hipSuccess)
    return fail(DEINFER_ERR_DEVICE, "prompt attention: LDS size refused");
  hipLaunchKernelGGL((prompt_tile_kernel<DT, KS, WAVES, FULL>), dim3((unsigned)pl.shares), dim3(C::THREADS), C::LDS, s, P);
  if (int rc = check_launch("prompt attention")) return rc;
  hipLaunchKernelGGL((prompt_join_kernel<DT, C::COLS, C::ROWS>), dim3((unsigned)pl.shares, C::ROWS / 16), dim3(256), 0, s, P);
  return check_launch("prompt attention");
}
template <int DT, int KS>
int launch_prompt_steps(const PromptPlan &pl, const PromptParams &P, hipStream_t s) {
  const bool full = P.head_dim == 16 * KS;
  if constexpr (KS <= 8)
    if (pl.rows == 256) return full ? launch_prompt_tiles<DT, KS, 8, true>(pl, P, s) : launch_prompt_tiles<DT, KS, 8, false>(pl, P, s);
  return full ? launch_prompt_tiles<DT, KS, 4, true>(pl, P, s) : launch_prompt_tiles<DT, KS, 4, false>(pl, P, s);
}
template <int DT, int DP>
int launch_prompt_rows(const PromptPlan &pl, const PromptParams &P, hipStream_t s) {
  if (P.head_dim == DP) hipLaunchKernelGGL((prompt_rows_kernel<DT, DP, true>), dim3((unsigned)pl.shares), dim3(ATT_THREADS), 0, s, P);
  else hipLaunchKernelGGL((prompt_rows_kernel<DT, DP, false>), dim3((unsigned)pl.shares), dim3(ATT_THREADS), 0, s, P);
  if (int rc = check_launch("prompt attention")) return rc;
  hipLaunchKernelGGL((prompt_join_kernel<DT, DP, 16>), dim3((unsigned)pl.shares), dim3(1024), 0, s, P);
  return check_launch("prompt attention");
}
template <int DT>
int launch_prompt(const PromptPlan &pl, const PromptParams &P, hipStream_t s) {
  const int D = P.head_dim;
  if (pl.rows == 16) return D <= 64 ? launch_prompt_rows<DT, 64>(pl, P, s) : D <= 128 ? launch_prompt_rows<DT, 128>(pl, P, s) : launch_prompt_rows<DT, 256>(pl, P, s);
  if (D <= 64) return launch_prompt_steps<DT, 4>(pl, P, s);
  if (D <= 80) return launch_prompt_steps<DT, 5>(pl, P, s);
  if (D <= 96) return launch_prompt_steps<DT, 6>(pl, P, s);
  if (D <= 128) return launch_prompt_steps<DT, 8>(pl, P, s);
  return launch_prompt_steps<DT, 16>(pl, P, s);
}

}  // namespace deinfer
