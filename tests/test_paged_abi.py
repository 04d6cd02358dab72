"""Host-side checks of the operators on a cache in pages: exported symbols, refusals, workspaces.  Every call here returns before any launch."""
import ctypes
import itertools
import os
import re

import numpy as np
import pytest
import torch

import paper_2404_09336_amd as span
from paper_2404_09336_amd import paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK = dict(batch=2, heads=8, kv_heads=2, head_dim=128, dtype_code=1, page_size=16, num_pages=10, table_pages=4)
FAR = 1 << 40  # a pointer that nobody follows


def desc(**kw):
    return paged.make_paged_desc(**{**OK, **kw})


def with_workspace(use, **kw):
    d = desc(**kw)
    d.workspace, d.workspace_bytes = FAR, paged.paged_workspace_bytes(d, use)
    return d


def call(name, d, *args):
    return getattr(paged._library(), name)(ctypes.byref(d) if d is not None else None, *args)


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "span_paged.h")).read()
    names = set(re.findall(r"\b(paged_\w+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S)))
    assert {"paged_append", "paged_decode_attn", "paged_span_decode_attn", "paged_prompt_attn", "paged_evict", "paged_workspace_bytes",
            "paged_workspace_init", "paged_check"} <= names
    for name in names:
        assert hasattr(paged._library(), name), name


SHAPES = [dict(batch=0), dict(batch=-1), dict(batch=65536), dict(heads=0), dict(kv_heads=0), dict(heads=7), dict(heads=34), dict(head_dim=96), dict(head_dim=0),
          dict(page_size=8), dict(page_size=48), dict(page_size=2048), dict(page_size=0), dict(num_pages=0), dict(num_pages=1 << 27), dict(table_pages=0),
          dict(table_pages=(1 << 18) + 1), dict(num_tokens=-1), dict(num_intervals=-1)]


@pytest.mark.parametrize("bad", SHAPES)
def test_shapes_are_refused(bad):
    d = desc(**bad)
    assert call("paged_check", d) == -2
    assert paged.paged_workspace_bytes(d, paged.PAGED_DECODE) == 0
    assert call("paged_append", d, *[FAR] * 9) == -2
    assert call("paged_decode_attn", d, *[FAR] * 5, 1.0, None, FAR) == -2
    assert call("paged_span_decode_attn", d, *[FAR] * 7, 1.0, None, FAR) == -2
    assert call("paged_prompt_attn", d, *[FAR] * 6, 1.0, FAR) == -2
    assert call("paged_evict", d, *[FAR] * 9) == -2
    assert call("paged_workspace_init", d) == -2


def test_types_and_missing_descriptors_are_refused():
    assert call("paged_check", desc(dtype_code=3)) == -3 and call("paged_check", None) == -1 and call("paged_check", desc()) == 0
    assert call("paged_decode_attn", None, *[FAR] * 5, 1.0, None, FAR) == -1
    assert call("paged_evict", desc(dtype_code=-1, budget=4), *[FAR] * 9) == -3
    for bad in (dict(window=-1), dict(sinks=1 << 31), dict(budget=-5), dict(recent=1 << 40), dict(num_splits=-1)):
        with pytest.raises(ValueError):
            desc(**bad)


def test_missing_pointers_are_refused():
    without = lambda n, i: [None if k == i else FAR for k in range(n)]  # noqa: E731
    for i in range(5):
        assert call("paged_decode_attn", with_workspace(paged.PAGED_DECODE), *without(5, i), 1.0, None, FAR) == -1
    assert call("paged_decode_attn", with_workspace(paged.PAGED_DECODE), *[FAR] * 5, 1.0, None, None) == -1
    d = with_workspace(paged.PAGED_SPAN_DECODE, num_intervals=3)
    for i in range(7):
        assert call("paged_span_decode_attn", d, *without(7, i), 1.0, None, FAR) == -1
    d = with_workspace(paged.PAGED_PROMPT, num_tokens=20)
    for i in range(6):
        assert call("paged_prompt_attn", d, *without(6, i), 1.0, FAR) == -1
    assert call("paged_prompt_attn", d, *[FAR] * 6, 1.0, None) == -1
    for i in range(6):
        assert call("paged_append", desc(num_tokens=2), *without(6, i), FAR, FAR, FAR) == -1
    d = with_workspace(paged.PAGED_EVICT, budget=8)
    for i in (0, 1, 2, 3, 4, 5, 6, 7, 8):
        assert call("paged_evict", d, *without(9, i)) == -1


def test_append_without_offsets_is_one_token_each():
    assert call("paged_append", desc(num_tokens=3), *[FAR] * 6, None, None, None) == -2
    assert call("paged_append", desc(num_tokens=0), *[None] * 9) == -2
    assert call("paged_append", desc(num_tokens=0), *[FAR] * 9) == 0  # nothing to do


def test_budgets_are_refused():
    for bad in (dict(budget=0), dict(budget=8, sinks=5, recent=4), dict(budget=8, sinks=2 ** 31 - 1, recent=2 ** 31 - 1)):
        d = desc(**bad)
        d.workspace, d.workspace_bytes = FAR, 1 << 30
        assert call("paged_evict", d, *[FAR] * 9) == -2


@pytest.mark.parametrize("use", range(6))
def test_workspaces_are_refused(use):
    """Missing, a byte short, misaligned."""
    d = desc(budget=20, table_pages=64, num_pages=200, num_intervals=4, num_tokens=100)
    need = paged.paged_workspace_bytes(d, use)
    assert need > 0 and need % 256 == 0
    run = {0: lambda: call("paged_decode_attn", d, *[FAR] * 5, 1.0, None, FAR), 1: lambda: call("paged_decode_attn", d, *[FAR] * 5, 1.0, FAR, FAR),
           2: lambda: call("paged_span_decode_attn", d, *[FAR] * 7, 1.0, None, FAR), 3: lambda: call("paged_span_decode_attn", d, *[FAR] * 7, 1.0, FAR, FAR),
           4: lambda: call("paged_prompt_attn", d, *[FAR] * 6, 1.0, FAR), 5: lambda: call("paged_evict", d, *[FAR] * 9)}[use]
    for at, size in ((None, need), (FAR, need - 1), (FAR + 64, need)):
        d.workspace, d.workspace_bytes = at, size
        assert run() == -4
    assert paged.paged_workspace_bytes(d, 6) == 0 and paged.paged_workspace_bytes(d, -1) == 0


def test_workspace_init_needs_the_counters():
    d = desc(batch=100, heads=16, kv_heads=16)
    for at, size in ((None, 1 << 20), (FAR, 100 * 16 * 4 - 1), (FAR + 16, 1 << 20)):
        d.workspace, d.workspace_bytes = at, size
        assert call("paged_workspace_init", d) == -4


def test_prompts_without_tokens_and_with_too_many():
    assert call("paged_prompt_attn", desc(num_tokens=0), None, *[FAR] * 5, 1.0, None) == 0
    assert call("paged_prompt_attn", desc(num_tokens=65536 * 32), *[FAR] * 6, 1.0, FAR) == -2  # tiles of 32 tokens of 4 heads: the grid's limit


def slices(lens, rooms, whole):
    """Slices of a dense call as the kernel finds them."""
    total = lambda T: sum(1 if n <= whole else -(-n // T) for n in lens)  # noqa: E731
    longest, T = max(max(lens), 1), max(max(lens), 1)
    if longest <= whole:
        return len(lens)
    for room in rooms:
        T = longest
        if room > len(lens):
            T = max(-(-int(sum(lens) / (room - 0.5 * len(lens))) // 32) * 32, 128)
            while T < longest and total(T) > room:
                T = min(max(-(-int(T * total(T) / room) // 32) * 32, -(-(T + T // 16) // 32) * 32), longest)
        if min(T, longest) * max(room, len(lens)) <= 1.4 * sum(lens) or T <= 128:
            break
    return total(T)


def test_the_grid_holds_every_slice():
    """The workspace has a state for every slice that any lengths give."""
    rng = np.random.default_rng(0)
    for B, KV, G, D, TP in itertools.product([1, 2, 17, 64, 200, 512], [1, 3, 8, 32], [1, 4], [64, 128], [9, 17, 40, 700]):
        d = desc(batch=B, heads=KV * G, kv_heads=KV, head_dim=D, table_pages=TP, num_pages=1 << 20)
        need = paged.paged_workspace_bytes(d, paged.PAGED_DECODE)
        if TP * 16 <= 256:
            assert need == 0                       # nothing to cut
            continue
        counters = -(-B * KV * 4 // 256) * 256
        rows = (need - counters) // (KV * G * (D + 2) * 4)
        rooms = max(1, 512 // KV), rows
        for lens in ([TP * 16] * B, [0] * B, [1] * (B - 1) + [TP * 16], [257] * B, list(rng.integers(0, TP * 16 + 1, B))):
            assert slices([int(n) for n in lens], rooms, 256) <= rows, (B, KV, TP)


def test_binding_refuses_host_tensors():
    pool = torch.zeros((4, 2, 16, 64))
    with pytest.raises(ValueError):
        span.paged_decode_attn(torch.zeros((1, 2, 64)), pool, pool, torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 1.0)
    with pytest.raises(ValueError):
        span.paged_append(torch.zeros((1, 2, 64)), torch.zeros((1, 2, 64)), pool, pool, torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError):
        span.paged_evict(pool, pool, torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros((1, 2, 32)), 4)
