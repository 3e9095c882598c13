// Products of at most sixteen rows, int8 operands, results scaled to 16 bits and gated.
#define ABFT_EPI abft::EPI_GATED
#define ABFT_SKINNY_NAME(what, out) launch_gated_##what##_##out
#include "gemm_scaled_skinny.inc"
