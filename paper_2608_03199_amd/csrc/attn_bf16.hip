// attn_bf16.hip -- the packed attention's kernels for bf16 values.
#include "attn_kernels.h"

hipError_t sieve::attn_launch_bf16(AttnKind kind, int dp, const AttnArgs& a, int grid,
                                 hipStream_t s) {
  return launch_type<bf16>(kind, dp, a, grid, s);
}
