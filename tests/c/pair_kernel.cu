// The kernel of CTA pairs by itself, for a look at what the compiler makes of it.
#include "kb_matmul.cuh"
template __global__ void kb::matmul_pair_kernel<false>(const __grid_constant__ CUtensorMap, const __grid_constant__ CUtensorMap,
                                                       const kb::MatmulParams);
template __global__ void kb::matmul_pair_kernel<true>(const __grid_constant__ CUtensorMap, const __grid_constant__ CUtensorMap,
                                                      const kb::MatmulParams);
static_assert(kb::PairTile::kRegsLaunch == 168, "the test looks for this number");
