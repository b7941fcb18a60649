// Attention of packed prompts (tq_sdpa_prompt): choice of the kernel.
#include "tq_prompt.cuh"

namespace tq {

cudaError_t launch_prompt(const PromptArgs& a, cudaStream_t st) { return launch_prompt_simple(a, st); }

}  // namespace tq
