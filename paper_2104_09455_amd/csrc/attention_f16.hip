// Attention over a paged cache, f16 queries.
#define ABFT_DT abft::DT_F16
#define ABFT_ATTENTION_NAME launch_attention_f16
#include "attention.inc"
