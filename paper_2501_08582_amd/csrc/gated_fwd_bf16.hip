// Whole-tile instances of the gated block's forward above rank 48: the kernel of
// fwd_bf16.hip over two projections, a workgroup's tile of the gate and then of the up
// projection (the slabs of two A's do not fit LDS beside the stages of 256 tokens x 256 features; see
// gated_pair_fwd_bf16.hip for the ranks where they do).
#define LORS_GATED 1
#include "fwd_bf16.hip"
