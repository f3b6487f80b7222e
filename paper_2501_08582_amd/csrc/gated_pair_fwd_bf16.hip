// Whole-tile instances of the gated block's forward up to rank 48: the kernel of
// fwd_bf16.hip with both projections in one tile.
//
// What bounds it: the main loop of fwd_kernel, whose K-step is the same, and the stores
// of its epilogue, which nothing overlaps (one workgroup fills a CU's LDS).  4096 tokens,
// 11008 x 4096, rank 16, with G and U kept: 747 us (993 TFLOP/s), serving 675; one tile after the
// other, with act(g) parked in H, 825.  777 tokens of 2744 x 1032, rank 24: 31 us
// against 51, since half as many columns to a tile give 192-token tiles for all CUs.
#define LORS_GATED 2
#include "fwd_bf16.hip"
