// attn_f16.hip -- the packed attention's kernels for f16 values.
#include "attn_kernels.h"

hipError_t sieve::attn_launch_f16(AttnKind kind, int dp, const AttnArgs& a, int grid,
                                 hipStream_t s) {
  return launch_type<f16>(kind, dp, a, grid, s);
}
