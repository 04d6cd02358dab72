"""Slices of one-token calls over 4-bit pages against their plan (host arithmetic that the kernels share), under AddressSanitizer + UBSan with plain g++."""
import os
import subprocess
import sys

import pytest

from paper_2404_09336_amd import paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_windowed_slices_have_their_rows(tmp_path):
    exe = tmp_path / "host_paged_fp4_plan"
    csrc = os.path.join(ROOT, "paper_2404_09336_amd", "csrc")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-static-libasan", "-static-libubsan", "-I" + os.path.join(ROOT, "include"), "-I" + csrc,
           os.path.join(ROOT, "tests", "host_paged_fp4_plan.cpp"), os.path.join(csrc, "paged_host.cpp"), "-o", str(exe)]
    subprocess.run(cmd, check=True)
    res = subprocess.run([str(exe)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    sys.stdout.write(res.stdout[-2000:])
    assert res.returncode == 0 and "host_paged_fp4_plan: ok" in res.stdout


@pytest.mark.parametrize("window,sinks,rows", [(4096, 0, 9), (4092, 4, 9), (2048, 0, 5), (1536, 0, 4), (1025, 0, 3), (1023, 1, 0), (1024, 0, 0), (1 << 30, 0, 63), (1 << 30, 64, 63)])
def test_the_workspace_of_a_window(window, sinks, rows):
    """One sequence, 32 query heads on 8 KV heads of 128, a table of 32000 positions: counters and a state for each slice of 512 positions of the units that the window can touch; none
    for up to 1024 positions, which are never cut."""
    d = paged.make_paged_desc(1, 32, 8, 128, 2, 16, 1 << 12, 2000, window=window, sinks=sinks)
    rounded = lambda n: -(-n // 256) * 256  # noqa: E731
    want = rounded(4 * 9) + rounded(rows * 32 * 2 * 4) + rounded(rows * 32 * 128 * 4) if rows else 0
    assert paged.paged_workspace_bytes(d, paged.PAGED_DECODE_FP4) == want
