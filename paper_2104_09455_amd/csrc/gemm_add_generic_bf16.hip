// Generic kernel, int8 operands, results scaled to bf16 and added to a residual.
#define ABFT_DT abft::DT_I8
#define ABFT_OUT abft::DT_BF16
#define ABFT_EPI abft::EPI_ADD
#define ABFT_FAMILY 3
#define ABFT_LAUNCH_NAME launch_add_generic_bf16
#include "gemm_launch.inc"
