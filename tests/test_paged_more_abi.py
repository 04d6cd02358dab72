"""Host-side checks of rotated and 4-bit appends, attention over 4-bit pages and page selection: refusals, workspaces.  Every call here returns before any launch."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2404_09336_amd as span
from paged_more_reference import from_fp4, place, pool_fp4, read_fp4, to_fp4
from paper_2404_09336_amd import paged
from test_paged_abi import FAR, SHAPES, call, desc, with_workspace

ROTATION = dict(table=FAR, positions=100, channels=64, paired=0)


def turn(**kw):
    r = {**ROTATION, **kw}
    return ctypes.byref(paged._Rotation(r["table"], r["positions"], r["channels"], r["paired"]))


def every_call(d):
    """(name, result) of every entry point, all pointers given."""
    yield "rotary", call("paged_append_rotary", d, turn(), *[FAR] * 11)
    yield "append", call("paged_append_fp4", d, turn(), *[FAR] * 10)
    yield "read", call("paged_read_fp4", d, *[FAR] * 7)
    yield "decode", call("paged_decode_attn_fp4", d, *[FAR] * 5, 1.0, FAR)
    yield "span", call("paged_span_decode_attn_fp4", d, *[FAR] * 7, 1.0, FAR)
    yield "select", call("paged_select", d, *[FAR] * 7)
    yield "selected", call("paged_selected_decode_attn", d, *[FAR] * 6, 1.0, FAR)


@pytest.mark.parametrize("bad", SHAPES)
def test_shapes_are_refused(bad):
    for name, rc in every_call(desc(budget=3, **bad)):
        assert rc == -2, name
    for use in (paged.PAGED_SELECT, paged.PAGED_SELECTED_DECODE, paged.PAGED_DECODE_FP4, paged.PAGED_SPAN_DECODE_FP4):
        assert paged.paged_workspace_bytes(desc(budget=3, **bad), use) == 0


def test_types_and_missing_descriptors_are_refused():
    for name, rc in every_call(desc(budget=3, dtype_code=3)):
        assert rc == -3, name
    for name, rc in every_call(None):
        assert rc == -1, name


@pytest.mark.parametrize("bad", [dict(channels=0), dict(channels=8), dict(channels=40), dict(channels=144), dict(channels=-16), dict(positions=0), dict(positions=-1),
                                 dict(table=FAR + 4)])
def test_rotations_are_refused(bad):
    d = desc(num_tokens=2)
    assert call("paged_append_rotary", d, turn(**bad), *[FAR] * 11) == -2
    assert call("paged_append_fp4", d, turn(**bad), *[FAR] * 10) == -2


def test_missing_pointers_are_refused():
    without = lambda n, i, rest: [None if k == i else FAR for k in range(n)] + rest  # noqa: E731
    d = desc(num_tokens=2)
    for i in range(6):
        assert call("paged_append_rotary", d, turn(), *without(6, i, [None] * 5)) == -1
        assert call("paged_append_fp4", d, None, *without(6, i, [None] * 4)) == -1
    assert call("paged_append_rotary", d, None, *[FAR] * 11) == -1
    assert call("paged_append_rotary", d, turn(table=None), *[FAR] * 11) == -1
    for q in ([FAR, None], [None, FAR]):  # one of q and q_out
        assert call("paged_append_rotary", d, turn(), *[FAR] * 6, None, None, None, *q) == -1
        assert call("paged_append_fp4", d, turn(), *[FAR] * 6, None, None, *q) == -1
    assert call("paged_append_fp4", desc(num_tokens=0), None, *[FAR] * 6, None, None, FAR, FAR) == 0  # q without a rotation
    for i in (0, 1, 2, 3, 5, 6):
        assert call("paged_read_fp4", d, *without(7, i, [])) == -1
    for i in range(5):
        assert call("paged_decode_attn_fp4", with_workspace(paged.PAGED_DECODE_FP4), *without(5, i, []), 1.0, FAR) == -1
    assert call("paged_decode_attn_fp4", with_workspace(paged.PAGED_DECODE_FP4), *[FAR] * 5, 1.0, None) == -1
    for i in range(7):
        assert call("paged_span_decode_attn_fp4", with_workspace(paged.PAGED_SPAN_DECODE_FP4, num_intervals=3), *without(7, i, []), 1.0, FAR) == -1
    for i in (0, 1, 2, 3, 4, 6):
        assert call("paged_select", with_workspace(paged.PAGED_SELECT, budget=3), *without(7, i, [])) == -1
    for i in range(6):
        assert call("paged_selected_decode_attn", with_workspace(paged.PAGED_SELECTED_DECODE, budget=3), *without(6, i, []), 1.0, FAR) == -1


def test_without_offsets_there_is_one_token_each_and_without_tokens_nothing_to_do():
    d = desc(num_tokens=3)
    assert call("paged_append_rotary", d, turn(), *[FAR] * 6, *[None] * 5) == -2
    assert call("paged_append_fp4", d, None, *[FAR] * 6, *[None] * 4) == -2
    assert call("paged_read_fp4", d, *[FAR] * 4, None, FAR, FAR) == -2
    d = desc(num_tokens=0)
    assert call("paged_append_rotary", d, turn(), *[None] * 11) == 0
    assert call("paged_append_fp4", d, None, *[None] * 10) == 0
    assert call("paged_read_fp4", d, *[None] * 7) == 0


def test_more_tokens_than_a_grid_holds():
    """2^31 waves: of 65535 heads of 128 channels, fp32, a row of K, V and q takes thousands."""
    d = desc(heads=65535, kv_heads=65535, batch=1, dtype_code=0, num_tokens=(1 << 31) - 1)
    assert call("paged_append_rotary", d, turn(), *[FAR] * 11) == -2
    assert call("paged_append_fp4", d, turn(), *[FAR] * 10) == -2
    assert call("paged_read_fp4", d, *[FAR] * 7) == -2


def test_more_waves_than_a_launch_numbers():
    """2^32 lanes: rows of 2^26 tokens take a wave each at least."""
    d = desc(heads=1, kv_heads=1, batch=1, dtype_code=1, num_tokens=(1 << 26) + 1)
    assert call("paged_append_rotary", d, turn(), *[FAR] * 11) == -2
    assert call("paged_append_fp4", d, turn(), *[FAR] * 10) == -2
    assert call("paged_read_fp4", d, *[FAR] * 7) == -2


@pytest.mark.parametrize("budget,sinks,recent,good", [(0, 0, 0, False), (1, 0, 0, True), (1, 0, 1, True), (1, 0, 2, False), (2, 0, 2, True), (2, 0, 17, True), (2, 0, 18, False),
                                                      (2, 1, 1, True), (2, 16, 1, True), (2, 17, 1, False), (3, 17, 1, True), (1 << 30, (1 << 31) - 1, (1 << 31) - 1, True)])
def test_what_always_stays_has_to_fit_the_list(budget, sinks, recent, good):
    """Pages of 16: the last `recent` positions can lie on floor((recent + 14) / 16) + 1 of them."""
    d = with_workspace(paged.PAGED_SELECT, budget=budget, sinks=sinks, recent=recent)
    assert (paged.paged_workspace_bytes(d, paged.PAGED_SELECT) > 0) == good
    d.workspace, d.workspace_bytes = None, 0
    assert call("paged_select", d, *[FAR] * 7) == (-4 if good else -2)
    if budget == 0:
        assert call("paged_selected_decode_attn", d, *[FAR] * 6, 1.0, FAR) == -2
        assert paged.paged_workspace_bytes(d, paged.PAGED_SELECTED_DECODE) == 0


@pytest.mark.parametrize("use", [paged.PAGED_SELECT, paged.PAGED_SELECTED_DECODE, paged.PAGED_DECODE_FP4, paged.PAGED_SPAN_DECODE_FP4])
def test_workspaces_are_refused(use):
    """Missing, a byte short, misaligned."""
    d = desc(budget=40, table_pages=200, num_pages=500, num_intervals=4)
    need = paged.paged_workspace_bytes(d, use)
    assert need > 0 and need % 256 == 0
    run = {paged.PAGED_SELECT: lambda: call("paged_select", d, *[FAR] * 7), paged.PAGED_SELECTED_DECODE: lambda: call("paged_selected_decode_attn", d, *[FAR] * 6, 1.0, FAR),
           paged.PAGED_DECODE_FP4: lambda: call("paged_decode_attn_fp4", d, *[FAR] * 5, 1.0, FAR),
           paged.PAGED_SPAN_DECODE_FP4: lambda: call("paged_span_decode_attn_fp4", d, *[FAR] * 7, 1.0, FAR)}[use]
    for at, size in ((None, need), (FAR, need - 1), (FAR + 64, need)):
        d.workspace, d.workspace_bytes = at, size
        assert run() == -4
    assert all(paged.paged_workspace_bytes(d, other) == 0 for other in (6, 7, 15, 20))


def test_selected_calls_are_cut_by_the_list():
    """A list of few positions asks for no workspace, whatever the table could hold."""
    assert paged.paged_workspace_bytes(desc(budget=16, table_pages=1000, num_pages=3000), paged.PAGED_SELECTED_DECODE) == 0
    assert paged.paged_workspace_bytes(desc(budget=17, table_pages=1000, num_pages=3000), paged.PAGED_SELECTED_DECODE) > 0


def test_tensors_on_the_host_are_refused():
    K = torch.zeros((4, 2, 16, 64))
    K4 = torch.zeros((4, 2, 16, 34), dtype=torch.uint8)
    table, ctx, q, new = torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros((1, 4, 64)), torch.zeros((1, 2, 64))
    for f in (lambda: span.paged_append_rotary(new, new, K, K, table, ctx, torch.zeros((8, 64))), lambda: span.paged_append_fp4(new, new, K4, K4, table, ctx),
              lambda: span.paged_read_fp4(K4, K4, table, ctx, k_rows=new, v_rows=new), lambda: span.paged_decode_attn_fp4(q, K4, K4, table, ctx, 1.0),
              lambda: span.paged_span_decode_attn_fp4(q, K4, K4, table, ctx, ctx, ctx, 1.0), lambda: span.paged_select(q, K, torch.zeros((4, 2, 2, 64)), table, ctx, 2),
              lambda: span.paged_selected_decode_attn(q, K, K, table, ctx, torch.zeros((1, 2, 1), dtype=torch.int32), 1.0)):
        with pytest.raises(ValueError):
            f()


def test_reference_rounding():
    """The reference itself: values of the grid stay, borders go to the even number, every value to the nearest."""
    x = np.zeros(32)
    x[:16] = [0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6]
    code, byte = to_fp4(x)
    assert code[:16].tolist() == list(range(16)) and byte.tolist() == [127]
    x[:8] = [7, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5]
    code, byte = to_fp4(x)
    assert code[:8].tolist() == [7, 0, 2, 2, 4, 4, 6, 6] and byte.tolist() == [127]
    x[0] = np.nextafter(7, 8)
    assert to_fp4(x)[1].tolist() == [128]
    rng = np.random.default_rng(0)
    x = rng.standard_normal((200, 64)) * 2.0 ** rng.integers(-60, 60, (200, 1))
    y = from_fp4(*to_fp4(x))
    unit = 2.0 ** (to_fp4(x)[1].astype(float) - 127).repeat(32, -1)
    grid = np.concatenate((-np.array([0.5, 1, 1.5, 2, 3, 4, 6]), [0, 0.5, 1, 1.5, 2, 3, 4, 6]))
    assert np.array_equal(np.abs(x - y), np.abs(x[..., None] - unit[..., None] * grid).min(-1))
    for bad in (np.inf, np.nan, 3e38):
        x[0, 0] = bad
        assert to_fp4(x)[1][0].tolist()[0] == 255
    assert to_fp4(np.zeros(32))[1].tolist() == [1]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows", [16, 64])
def test_reference_layout(D, rows):
    """Every byte of a page is one row's, and what is written is read back."""
    for is_v in (False, True):
        at = np.concatenate([np.concatenate(place(rows, D, r, is_v)) for r in range(rows)])
        assert np.array_equal(np.sort(at), np.arange(rows * (D // 2 + D // 32)))
        x = np.random.default_rng(1).standard_normal((3, 2, rows, D))
        assert np.array_equal(read_fp4(pool_fp4(x, is_v), is_v), from_fp4(*to_fp4(x)))
