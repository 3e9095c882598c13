// All of a workgroup's k at once, int8 operands, results scaled to f16 and added to a residual.
#define ABFT_OUT abft::DT_F16
#define ABFT_EPI abft::EPI_ADD
#define ABFT_LAUNCH_NAME launch_joint_add_f16
#include "gemm_joint.inc"
