"""Rows of batches without q_start, with several tokens to a row: the kernels' own mapping (csrc/rows.h, compiled for the
host) and the library's sizes against the header's rule. No GPU."""
import ctypes
import shutil
import subprocess
from pathlib import Path

import pytest

from attention_oracle import Rows
from paper_2005_04091_amd import attention as A

ROOT = Path(__file__).resolve().parent.parent
P = 4096  # an aligned address; nothing is read there

DRIVER = """
#include <cstdio>
#include "rows.h"
int main(int n, char **) {
    for (int B : {1, 2, 3, 15, 16, 17, 64, 200})
        for (int q : {1, 2, 3, 8, 16, 128}) {
            const int rows = q == 1 ? B : B / q + B;
            for (int r = 0; r < rows; ++r) std::printf("%d %d %d %d\\n", B, q, r, sequence_of_row(r, q, B));
        }
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_rows_of_single_tokens(tmp_path):
    src = tmp_path / "rows.cpp"
    src.write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I",
                    str(ROOT / "paper_2005_04091_amd" / "csrc"), str(src), "-o", str(tmp_path / "rows")], check=True)
    got = {}
    for line in subprocess.run([str(tmp_path / "rows")], check=True, capture_output=True, text=True).stdout.splitlines():
        B, q, r, b = map(int, line.split())
        got.setdefault((B, q), {})[r] = b
    assert len(got) == 48
    for (B, q), rows in got.items():
        want = Rows(None, [5] * B, B, q)
        assert len(rows) == want.rows == library_rows(B, q)
        for r, b in rows.items():
            assert b == (want.of[r][0] if r in want.of else -1), (B, q, r)


def single(B, q_block):
    return A.spconv_batch(B, 16, 1000, q_block, B, 5000, 1000, P, P, None)


def library_rows(B, q_block):
    n = ctypes.c_int64()
    assert A._lib.spconv_batch_rows(single(B, q_block), n) == A.SPCONV_OK
    return n.value


def workspace(B, q_block, keep):
    n = ctypes.c_int64()
    assert A._lib.spconv_attention_workspace(2, single(B, q_block), 8, 2, 128, keep, n) == A.SPCONV_OK
    return n.value


@pytest.mark.parametrize("B", [1, 3, 64, 100])
@pytest.mark.parametrize("q_block", [2, 16, 64, 128])
def test_without_lists_single_tokens_are_planned_alike(B, q_block):
    """What q_block says is of no matter then: the same items, and so the same workspace."""
    assert workspace(B, q_block, 0) == workspace(B, 1, 0)


def test_rows_of_single_tokens_are_small():
    """Four pairs a row, however many tokens q_block would allow: partial outputs of tiles of 16."""
    assert workspace(16, 128, 64) == workspace(16, 1, 64) > 0
