"""Few rows of large weights beyond 8192 values of k, where K ends inside of the last k tile of a wavefront that has two tiles fewer than the
kernel is made for (results, flags and the other schemes' bits; where it reads is test_few_rows_reads.py's)."""
import pytest

import test_gpu_add_gated as block

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["add", "gated"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,N,K", [(4, 4096, 8208), (16, 2300, 9072), (1, 2600, 10256), (16, 4096, 10944), (9, 3100, 12304), (3, 3300, 13168), (2, 4096, 15152), (1, 3805, 15216)])
def test_k_ends_inside_of_the_shortest_wavefront_s_last_tile(M, N, K, dtype, kind):
    block.test_few_rows_of_large_weights(M, N, K, dtype, kind)
