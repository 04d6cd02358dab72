"""Plans, workspaces and counters of the calls on a cache in pages (host arithmetic), the plans under AddressSanitizer + UBSan with plain g++."""
import ctypes
import itertools
import os
import subprocess
import sys

import pytest

from paper_2404_09336_amd import paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_plans_of_one_token_calls(tmp_path):
    exe = tmp_path / "host_paged_plan"
    csrc = os.path.join(ROOT, "paper_2404_09336_amd", "csrc")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-static-libasan", "-static-libubsan", "-I" + os.path.join(ROOT, "include"), "-I" + csrc,
           os.path.join(ROOT, "tests", "host_paged_plan.cpp"), os.path.join(csrc, "paged_host.cpp"), "-o", str(exe)]
    subprocess.run(cmd, check=True)
    res = subprocess.run([str(exe)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    sys.stdout.write(res.stdout[-2000:])
    assert res.returncode == 0 and "host_paged_plan: ok" in res.stdout
