// Products of at most sixteen rows, int8 operands, results scaled to 16 bits.
#define ABFT_EPI abft::EPI_SCALE
#define ABFT_SKINNY_NAME(what, out) launch_scaled_##what##_##out
#include "gemm_scaled_skinny.inc"
