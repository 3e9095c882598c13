// Products of at most sixteen rows, int8 operands, results scaled to 16 bits.
#include "gemm_configs.h"
#include "gemm_skinny.h"

namespace abft {
namespace {

typedef void (*SkinnyKernel)(const GemmArgs);
template <int OUT, bool INJ>
SkinnyKernel skinny_kernel(int mode, int tn, bool bytes) {
    if (mode == MODE_NONE)
        return bytes ? gemm_skinny_kernel<DT_I8, 1, MODE_NONE, true, INJ, OUT> : gemm_skinny_kernel<DT_I8, 1, MODE_NONE, false, INJ, OUT>;
    if (tn == 1)
        return bytes ? gemm_skinny_kernel<DT_I8, 1, MODE_THREAD, true, INJ, OUT> : gemm_skinny_kernel<DT_I8, 1, MODE_THREAD, false, INJ, OUT>;
    return bytes ? gemm_skinny_kernel<DT_I8, 2, MODE_THREAD, true, INJ, OUT> : gemm_skinny_kernel<DT_I8, 2, MODE_THREAD, false, INJ, OUT>;
}

template <int OUT>
hipError_t launch(int mode, bool bytes, int columns, const GemmArgs& args, hipStream_t stream) {
    static_assert(skinny_lds_bytes(2) <= 64 * 1024, "more would have to be asked for");
    const int tn = mode == MODE_NONE || !args.report ? 1 : columns / 16;
    const SkinnyKernel kern = args.f_row >= 0 ? skinny_kernel<OUT, true>(mode, tn, bytes) : skinny_kernel<OUT, false>(mode, tn, bytes);
    const int tiles = (args.N + 16 * tn - 1) / (16 * tn);
    hipLaunchKernelGGL(kern, dim3((unsigned)tiles), dim3(64 * SKINNY_WAVES), skinny_lds_bytes(tn), stream, args);
    return hipGetLastError();
}

// rows not quantised yet (p.A: of the output's type; no report, no planted fault)
template <int OUT>
hipError_t launch_few(int mode, bool bytes, const GemmArgs& args, hipStream_t stream) {
    static_assert(skinny_lds_bytes(1) + SKINNY_FEW_BYTES <= 64 * 1024, "more would have to be asked for");
    if (args.report || args.f_row >= 0 || !skinny_few_fits(args.M, args.K)) return hipErrorInvalidValue;  // (never picked)
    SkinnyKernel kern;
    if (mode == MODE_NONE) kern = bytes ? gemm_skinny_kernel<DT_I8, 1, MODE_NONE, true, false, OUT, true> : gemm_skinny_kernel<DT_I8, 1, MODE_NONE, false, false, OUT, true>;
    else kern = bytes ? gemm_skinny_kernel<DT_I8, 1, MODE_THREAD, true, false, OUT, true> : gemm_skinny_kernel<DT_I8, 1, MODE_THREAD, false, false, OUT, true>;
    hipLaunchKernelGGL(kern, dim3((unsigned)((args.N + 15) / 16)), dim3(64 * SKINNY_WAVES), skinny_lds_bytes(1) + skinny_few_bytes(args.M, args.K), stream, args);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_scaled_few_f16(int mode, bool bytes, const GemmArgs& args, hipStream_t stream) {
    return launch_few<DT_F16>(mode, bytes, args, stream);
}
hipError_t launch_scaled_few_bf16(int mode, bool bytes, const GemmArgs& args, hipStream_t stream) {
    return launch_few<DT_BF16>(mode, bytes, args, stream);
}
hipError_t launch_scaled_skinny_f16(int mode, bool bytes, int columns, const GemmArgs& args, hipStream_t stream) {
    return launch<DT_F16>(mode, bytes, columns, args, stream);
}
hipError_t launch_scaled_skinny_bf16(int mode, bool bytes, int columns, const GemmArgs& args, hipStream_t stream) {
    return launch<DT_BF16>(mode, bytes, columns, args, stream);
}

}  // namespace abft
