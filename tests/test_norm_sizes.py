"""The norm's choice of a kernel, by its own rule compiled for the host: rows of up to 2^31 - 1 values, where a sum that passes an int is no
constant expression and does not compile."""
import subprocess

import pytest

from paper_2104_09455_amd import build


@pytest.mark.parametrize("k,chunks", [(1, 1), (2048, 1), (2049, 2), (8192, 4), (8193, 5), (2 ** 31 - 2048, 1048575), (2 ** 31 - 2047, 1048576), (2 ** 31 - 1, 1048576)])
def test_chunks_that_a_thread_holds(k, chunks, tmp_path):
    src = tmp_path / "sizes.hip"
    src.write_text(f'#include "rms_norm.hip"\nstatic_assert(held_chunks({k}) == {chunks}, "chunks");\n')
    r = subprocess.run([build.HIPCC, *build.FLAGS, "-I", build.CSRC, "--offload-host-only", "-fsyntax-only", str(src)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
