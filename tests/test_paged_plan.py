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


def counters(batch, kv_heads):
    """Bytes of the tickets of every (sequence, KV head) and of every sequence."""
    return -(-4 * batch * (kv_heads + 1) // 256) * 256


def rounded(n):
    return -(-n // 256) * 256


@pytest.mark.parametrize("batch,kv_heads", [(1, 1), (3, 5), (100, 16), (512, 1), (65535, 1)])
def test_the_least_workspace_with_counters(batch, kv_heads):
    """A byte less is refused by everything that has tickets; as much is what an eviction of short tables asks for."""
    d = paged.make_paged_desc(batch, kv_heads, kv_heads, 128, 1, 16, 10, 4, budget=9)
    assert paged.paged_workspace_bytes(d, paged.PAGED_EVICT) == counters(batch, kv_heads)
    lib, far = paged._library(), 1 << 40  # a pointer that nobody follows
    for size in (0, 4 * batch * kv_heads, counters(batch, kv_heads) - 1):
        d.workspace, d.workspace_bytes = far, size
        assert lib.paged_workspace_init(ctypes.byref(d)) == -4
        assert lib.paged_evict(ctypes.byref(d), *[far] * 9) == -4


def test_the_workspace_holds_a_state_of_every_slice_and_no_more():
    """Of a dense one-token call on 256 positions and more: the counters, then (maximum, sum) and outputs of every query head of as many slices as the grid has rows."""
    for B, KV, G, D, TP in itertools.product([1, 2, 17, 64, 200, 512], [1, 3, 8, 32], [1, 4], [64, 128], [17, 40, 700]):
        d = paged.make_paged_desc(B, KV * G, KV, D, 1, 16, 1 << 20, TP)
        rows = max(B, min(max(1, 1024 // KV), -(-TP * 16 // 128) * B))
        states = rows * KV * G
        want = counters(B, KV) + rounded(states * 2 * 4) + rounded(states * D * 4)
        assert paged.paged_workspace_bytes(d, paged.PAGED_DECODE) == want, (B, KV, G, D, TP)
        capacity = TP * 16
        with_weights = want + rounded(B * KV * G * 2 * 4) + rounded(B * KV * G * capacity * 4)
        assert paged.paged_workspace_bytes(d, paged.PAGED_DECODE_WEIGHTS) == with_weights
