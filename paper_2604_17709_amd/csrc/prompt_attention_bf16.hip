// Attention over packed keys and values in bf16.
#include "prompt_attention_launch.h"

namespace deinfer {

int launch_prompt_bf16(const PromptPlan &pl, const PromptParams &P, hipStream_t s) { return launch_prompt<DT_BF16>(pl, P, s); }

}  // namespace deinfer
