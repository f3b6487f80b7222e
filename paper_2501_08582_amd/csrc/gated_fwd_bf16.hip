// Whole-tile instances of the gated block's forward: the kernel of fwd_bf16.hip over
// two projections.
//
// What bounds it: see fwd_kernel; a workgroup runs that kernel's main loop twice.  Two
// tiles to a workgroup, one after the other, and not one tile of 128 + 128 interleaved
// features: the slabs of two A's do not fit LDS beside the stages above rank 48.
#define LORS_GATED 1
#include "fwd_bf16.hip"
