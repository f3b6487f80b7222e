// Thin-tile instances of the gated block's dX (see dx_thin_bf16.hip and
// gated_dx_bf16.hip).
#define LORS_GATED 1
#define LORS_THIN_TILES 1
#define LORS_COPY_WAIT "s_nop 3"
#include "dx_bf16.hip"
