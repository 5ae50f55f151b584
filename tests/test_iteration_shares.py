"""How the attention kernels share out keys, where the host can compute it (compiled from the kernels' own header)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_pieces_of_more_work_than_32_bits_count(tmp_path):
    """The longest chunks at the longest positions: the length of a piece, which the kernel holds in 32 bits, must not wrap around to a short one, of which
    there would be more than the workspace has parts for."""
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    shares = [0, 1, 511, 512, 513, 512 << 20, 512 * ((1 << 24) - 1), 512 << 24, 512 << 31, 512 * ((1 << 32) + 1), 1 << 55]
    (tmp_path / "p.cpp").write_text("#include <cstdio>\n#include <cstdlib>\n#include \"gnr_iter_internal.h\"\n"
                                    "int main(int n, char **a) { for (int i = 1; i < n; ++i) std::printf(\"%d\\n\", gnr::blocks_of_a_piece(std::atoll(a[i]), 512)); }\n")
    subprocess.run(["g++", "-std=c++17", f"-I{ROOT}/include", f"-I{ROOT}/paper_2602_02987_amd/csrc_iter", str(tmp_path / "p.cpp"), "-o", str(tmp_path / "p")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "p")] + [str(x) for x in shares], capture_output=True, text=True, check=True).stdout.split()]
    longest = (1 << 30) // 64                                       # blocks of keys of one request
    for share, size in zip(shares, got):
        assert size >= 1 and size * 512 >= min(share, longest * 512), (share, size)
        assert size == max(1, -(-share // 512)) or size > longest
        grown = size
        for _ in range(6):                                          # (the kernel lengthens it a few times)
            grown += grown // 8 + 1
        assert grown + longest < 1 << 31
