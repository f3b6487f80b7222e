// Adapter gradients of a gated block's two projections in one grid: the kernel of
// g_bf16.hip.
#define LORS_GATED 1
#include "g_bf16.hip"
