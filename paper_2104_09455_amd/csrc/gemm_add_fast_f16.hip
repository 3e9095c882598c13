// Direct-to-LDS kernel, int8 operands, results scaled to f16 and added to a residual.
#define ABFT_DT abft::DT_I8
#define ABFT_OUT abft::DT_F16
#define ABFT_EPI abft::EPI_ADD
#define ABFT_FAMILY 1
#define ABFT_LAUNCH_NAME launch_add_fast_f16
#include "gemm_launch.inc"
