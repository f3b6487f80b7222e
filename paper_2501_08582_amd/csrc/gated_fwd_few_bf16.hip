// The gated block's forward for few tokens: the kernel of fwd_few_bf16.hip over two
// projections, one launch.
#define LORS_GATED 1
#include "fwd_few_bf16.hip"
