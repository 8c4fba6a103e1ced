// Attention of many tokens: the kernels for heads of 64 values.
#include "tq_prompt.hpp"

namespace tq {

hipError_t launch_prompt_64(const PromptArgs &a, bool bf16, hipStream_t s) { return launch_prompt_d<64>(a, bf16, s); }

}  // namespace tq
