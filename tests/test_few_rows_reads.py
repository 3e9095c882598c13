"""Where the kernel of register-held activations reads weights: its own rule, compiled for the host, over every K that it takes."""
import subprocess

from paper_2104_09455_amd import build

SOURCE = """
#include <cstdio>
#include "gemm_configs.h"
using namespace abft;
int main() {
    int values = 0, wrong = 0;
    for (int K = 16; K <= 16384 + 1024; K += 16) {   // (rows come in 16-byte chunks)
        if (!resident_fits(1, K)) continue;
        ++values;
        const int T = resident_tiles(K), nkt = (K + 127) / 128;
        bool bad = resident_first(nkt, 0) != 0 || resident_first(nkt, 8) != nkt;
        for (int wave = 0; wave < 8; ++wave) {
            const int first = resident_first(nkt, wave), own = resident_first(nkt, wave + 1) - first;
            if (own < 0 || own > T) bad = true;
            for (int t = 0; t < T; ++t)
                for (int chunk = 0; chunk < 128; chunk += 16) {
                    const int k = first * 128 + t * 128 + chunk, at = first * 128 + resident_at(T, t, chunk, K - first * 128);
                    if (at < 0 || at + 16 > K) bad = true;                    // inside the row
                    if (t < own && k < K && at != k) bad = true;   // and what is wanted, where there is any
                }
        }
        if (bad) {
            ++wrong;
            std::printf("K = %d: %d tiles\\n", K, T);
        }
    }
    std::printf("%d of %d\\n", wrong, values);
    return 0;
}
"""


def test_no_read_leaves_the_row(tmp_path):
    src, exe = tmp_path / "reads.hip", tmp_path / "reads"
    src.write_text(SOURCE)
    subprocess.run([build.HIPCC, *build.FLAGS, "-I", build.CSRC, "--offload-host-only", str(src), "-o", str(exe)], check=True, capture_output=True, timeout=300)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True, timeout=60).stdout
    assert out.split("\n")[-2] == "0 of 992", out
