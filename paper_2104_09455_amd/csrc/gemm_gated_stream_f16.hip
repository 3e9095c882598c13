// Streaming kernel, int8 operands, results scaled to f16 and gated.
#define ABFT_DT abft::DT_I8
#define ABFT_OUT abft::DT_F16
#define ABFT_EPI abft::EPI_GATED
#define ABFT_FAMILY 2
#define ABFT_LAUNCH_NAME launch_gated_stream_f16
#include "gemm_launch.inc"
