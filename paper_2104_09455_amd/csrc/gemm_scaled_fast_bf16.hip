// Direct-to-LDS kernel, int8 operands, results scaled to bf16.
#define ABFT_DT abft::DT_I8
#define ABFT_OUT abft::DT_BF16
#define ABFT_FAMILY 1
#define ABFT_LAUNCH_NAME launch_scaled_fast_bf16
#include "gemm_launch.inc"
