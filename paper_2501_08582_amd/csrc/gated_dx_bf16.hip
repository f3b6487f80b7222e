// Whole-tile instances of the gated block's dX = dG . Wg' + dU . Wu': the kernel of
// dx_bf16.hip over two projections.
//
// What bounds it: dx_kernel's main loop, run twice.  4096 tokens, 13824 x 5120, rank 64: 1200 us
// (0.97 PFLOP/s) for 256 whole tiles and 64 in four pieces each, 919 + 462 with thin tiles in the
// pieces' place.  Two sums in one set of accumulators need no second pass over dX and one
// rounding.
#define LORS_GATED 1
#include "dx_bf16.hip"
