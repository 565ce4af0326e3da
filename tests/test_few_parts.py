"""Where the kernels of few rows load their weights from (csrc/gdn_few_parts.h), on the host: no load that they issue may reach past the weight's last row,
however a buffer load compares its scalar offset (k) with the bytes that its descriptor has: not at all, added to the lane's offset, or taken off
the bytes, in 32 bits that wrap."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "gdn_few_parts.h"
using namespace gdn::few;
int main(int argc, char** argv) {
    const int WR = atoi(argv[1]), gated = atoi(argv[2]);
    const int loads = WR / 8, half = (loads + 1) / 2, outs = gated ? WR / 2 : WR;
    const char* const w = reinterpret_cast<const char*>((uintptr_t)1 << 40);
    long long live = 0;
    for (int K = 64; K <= 448; K += 192)
        for (int64_t ld = K; ld <= K + 24; ld += 24)
            for (int N = 1; N <= 100; ++N) {
                const char* const end = w + ((int64_t)(N - 1) * ld + K) * 2;
                for (int n0 = 0; n0 < N; n0 += outs)
                    for (int j = 0; j < loads; ++j) {
                        // (the second weight's rows of a gated product begin at n0 too)
                        const Part p = rows_from(w, ld, N, K, j < half || gated ? n0 : n0 + 8 * half, WR);
                        for (int row = 0; row < 8; ++row)
                            for (int pos = 0; pos < 8; ++pos)
                                for (int k = 0; k < 2 * K; k += 2 * STEP) {
                                    const int off = load_offset(8 * j + row, 8 * (j >= half ? j - half : j) + row, pos, p.pitch);
                                    const bool cut[3] = {off >= p.bytes, (int64_t)off + k >= p.bytes, (uint32_t)off >= (uint32_t)p.bytes - (uint32_t)k};
                                    const char* const at = p.at + off + k;
                                    for (int way = 0; way < 3; ++way)
                                        if (!cut[way] && (at < w || at + 16 > end)) {
                                            std::printf("K %d ld %lld N %d outputs from %d, load %d row %d piece %d, %d bytes on: past the end (comparison %d)\n", K, (long long)ld, N, n0, j, row, pos, k, way);
                                            return 1;
                                        }
                                    // a row that is an output's has to be there, in its place
                                    const int r = n0 + 8 * (gated && j >= half ? j - half : j) + row;
                                    if (r < N && (cut[0] || cut[1] || cut[2] || at < w + (r * ld) * 2 + k || at >= w + (r * ld) * 2 + k + 2 * STEP)) {
                                        std::printf("K %d ld %lld N %d: row %d is not where it should be\n", K, (long long)ld, N, r);
                                        return 1;
                                    }
                                    live += !cut[1];
                                }
                    }
            }
    std::printf("%lld\n", live);
    return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    at = tmp_path_factory.mktemp("few_parts")
    (at / "parts.cpp").write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2605_05219_amd", "csrc"), str(at / "parts.cpp"), "-o", str(at / "parts")])
    return str(at / "parts")


@pytest.mark.parametrize("rows_of_weights,gated", [(8, 0), (16, 0), (32, 0), (16, 1), (32, 1)])
def test_no_load_reaches_past_the_weights(program, rows_of_weights, gated):
    res = subprocess.run([program, str(rows_of_weights), str(gated)], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout
    assert int(res.stdout) > 0
