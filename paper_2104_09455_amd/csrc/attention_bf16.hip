// Attention over a paged cache, bf16 queries.
#define ABFT_DT abft::DT_BF16
#define ABFT_ATTENTION_NAME launch_attention_bf16
#include "attention.inc"
