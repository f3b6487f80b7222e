// Adapter gradients of a gated block's two projections in one grid: the kernel of
// g_bf16.hip.
//
// What bounds it: g_kernel's main loop; one grid leaves one short last wave in place of two.
// 4096 tokens, 13824 x 5120, rank 64: 1077 to 1100 us (1.05 to 1.08 PFLOP/s).
#define LORS_GATED 1
#include "g_bf16.hip"
