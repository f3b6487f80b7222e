// Whole-tile instances of the gated block's dX = dG . Wg' + dU . Wu': the kernel of
// dx_bf16.hip over two projections.
#define LORS_GATED 1
#include "dx_bf16.hip"
