"""Checked kernels really multiply twice: a scaled product under the thread-level scheme issues every matrix instruction of the unprotected
one and as many redundant ones.  Planted faults cannot show this, since they flip a bit behind the products; the kernels' own assembly,
compiled here, does."""
import re
import subprocess

import pytest

from paper_2104_09455_amd import build


def tiled(kernel, cfgs, rest):
    return [tuple(f"{kernel}<ScaledCfg<CfgOf<DT_I8, {c}>::type, {out}, {epi}>, {rest(c, mode)}>" for mode in ("MODE_NONE", "MODE_THREAD"))
            for c, out, epi in cfgs]


CONFIGS = [("DT_F16", "EPI_ADD"), ("DT_BF16", "EPI_GATED")]
# (headers, the argument's type, pairs of an unprotected kernel and its checked form)
FAMILIES = {
    "joint": ("gemm_joint.h", "GemmArgs", [tuple(f"gemm_joint_kernel<{out}, {epi}, {layout}, {c}>" for c in ("false", "true"))
                                           for out, epi in CONFIGS for layout in ("JOINT_NK", "JOINT_NK_BYTES", "JOINT_KN")]),
    "resident": ("gemm_resident.h", "ResidentArgs", [tuple(f"gemm_resident_kernel<{out}, {epi}, {t}, {c}, {f}>" for c in ("false", "true"))
                                                     for out, epi in CONFIGS for t in (1, 5, 10) for f in ("false", "true")]),
    "skinny": ("gemm_skinny.h", "GemmArgs", [tuple(f"gemm_skinny_kernel<DT_I8, 1, {m}, {by}, false, {out}, {few}, {epi}>" for m in ("MODE_NONE", "MODE_THREAD"))
                                             for out, epi in CONFIGS + [("DT_F16", "EPI_SCALE")] for by in ("false", "true") for few in ("false", "true")]),
    "stream": ("gemm_stream.h", "GemmArgs", tiled("gemm_stream_kernel", [("CFG_S32", "DT_F16", "EPI_SCALE"), ("CFG_S32W", "DT_F16", "EPI_ADD"), ("CFG_S64", "DT_BF16", "EPI_GATED"), ("CFG_S128", "DT_F16", "EPI_ADD")],
                                                  lambda c, m: f"CfgOf<DT_I8, {c}>::NSTAGE, CfgOf<DT_I8, {c}>::KWAYS, {m}, false, false, false")),
    "fast": ("gemm_fast.h", "GemmArgs", tiled("gemm_fast_kernel", [("CFG_F128", "DT_F16", "EPI_ADD"), ("CFG_F128T", "DT_BF16", "EPI_GATED"), ("CFG_F64T", "DT_F16", "EPI_SCALE")],
                                              lambda c, m: f"CfgOf<DT_I8, {c}>::NSTAGE, {m}, false, false")),
    "generic": ("gemm_kernel.h", "GemmArgs", tiled("gemm_kernel", [("CFG_G128", "DT_F16", "EPI_ADD"), ("CFG_G64", "DT_BF16", "EPI_GATED"), ("CFG_G64K", "DT_F16", "EPI_SCALE"), ("CFG_G16", "DT_BF16", "EPI_GATED")],
                                                   lambda c, m: f"{m}, false, false, CfgOf<DT_I8, {c}>::KWAYS, LD_TURN")),
}


@pytest.mark.parametrize("family", FAMILIES)
def test_every_product_of_a_checked_kernel_is_issued_twice(family, tmp_path):
    header, args, pairs = FAMILIES[family]
    kernels = [k for pair in pairs for k in pair]
    src, asm = tmp_path / "all.hip", tmp_path / "all.s"
    src.write_text(f'#include "gemm_configs.h"\n#include "{header}"\nnamespace abft {{\n'
                   + "".join(f"template __global__ void {k}(const {args});\n" for k in kernels) + "}\n")
    subprocess.run([build.HIPCC, *build.FLAGS, "-I", build.CSRC, "--cuda-device-only", "-S", str(src), "-o", str(asm)], check=True,
                   capture_output=True, timeout=600)
    counts = []   # of the functions, in the order in which they are instantiated
    for line in asm.read_text().splitlines():
        if re.match(r"\t\.type\t\w+,@function", line):
            counts.append(0)
        elif re.match(r"\tv_mfma_i32", line):
            counts[-1] += 1
    assert len(counts) == len(kernels)
    wrong = [(k, plain, checked) for k, plain, checked in zip(kernels[1::2], counts[::2], counts[1::2]) if plain == 0 or checked != 2 * plain]
    assert not wrong
