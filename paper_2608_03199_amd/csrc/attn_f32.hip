// attn_f32.hip -- the packed attention's kernels for f32 values.
#include "attn_kernels.h"

hipError_t sieve::attn_launch_f32(AttnKind kind, int dp, const AttnArgs& a, int grid,
                                 hipStream_t s) {
  return launch_type<float>(kind, dp, a, grid, s);
}
