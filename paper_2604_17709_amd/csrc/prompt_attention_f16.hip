// Attention over packed keys and values in fp16.
#include "prompt_attention_launch.h"

namespace deinfer {

int launch_prompt_f16(const PromptPlan &pl, const PromptParams &P, hipStream_t s) { return launch_prompt<DT_F16>(pl, P, s); }

}  // namespace deinfer
