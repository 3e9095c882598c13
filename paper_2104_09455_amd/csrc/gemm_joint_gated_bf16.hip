// All of a workgroup's k at once, int8 operands, results scaled to bf16 and gated.
#define ABFT_OUT abft::DT_BF16
#define ABFT_EPI abft::EPI_GATED
#define ABFT_LAUNCH_NAME launch_joint_gated_bf16
#include "gemm_joint.inc"
