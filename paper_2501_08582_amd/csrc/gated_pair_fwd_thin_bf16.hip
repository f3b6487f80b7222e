// Thin-tile instances of the gated block's forward up to rank 48 (see fwd_thin_bf16.hip
// and gated_pair_fwd_bf16.hip).
#define LORS_GATED 2
#define LORS_THIN_TILES 1
#include "fwd_bf16.hip"
