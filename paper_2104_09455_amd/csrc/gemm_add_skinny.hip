// Products of at most sixteen rows, int8 operands, results scaled to 16 bits and added to a residual.
#define ABFT_EPI abft::EPI_ADD
#define ABFT_SKINNY_NAME(what, out) launch_add_##what##_##out
#include "gemm_scaled_skinny.inc"
