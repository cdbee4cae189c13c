// The kernels of prompts alone, for what the compiler says about them.
#include "kb_prompt.cuh"

#define KB_ONE(DT, DP)                                                                                                  \
  template __global__ void kb::attention_kernel<DT, DP>(const __grid_constant__ CUtensorMap, const __grid_constant__ CUtensorMap, \
                                                        const __grid_constant__ CUtensorMap, const kb::PromptParams);
KB_ONE(KB_F16, 64)
KB_ONE(KB_F16, 128)
KB_ONE(KB_BF16, 64)
KB_ONE(KB_BF16, 128)
