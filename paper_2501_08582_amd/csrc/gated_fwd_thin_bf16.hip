// Thin-tile instances of the gated block's forward (see fwd_thin_bf16.hip and
// gated_fwd_bf16.hip).
#define LORS_GATED 1
#define LORS_THIN_TILES 1
#define LORS_COPY_WAIT "s_nop 3"
#include "fwd_bf16.hip"
