"""Sequences that outgrow their block table: the new rows that have no place are dropped, none of the others is touched, and tokens keep their positions."""
import numpy as np
import pytest
import torch

import paper_2404_09336_amd as span
from paged_reference import DTYPES, Pages, attend

pytestmark = pytest.mark.gpu
TOL = 1e-5  # as for the other one-token and fp32 prompt calls


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ctx,new", [([65, 64, 30], None), ([2 ** 31 - 1, 66, -4], None), ([66, 64, 3], [5, 2, 3]), ([100, 2 ** 31 - 1, 65], [40, 3, 65])])
def test_append_past_the_table(dtype, ctx, new, gpu_device):
    """One row, and chunks whose beginning still fits, whose end does not, or both; positions are noted for rows that have a place only."""
    pages = Pages([64, 64, 64], 2, 2, 64, 16, dtype, gpu_device, seed=3)
    t = new or [1, 1, 1]
    off = np.cumsum([0] + t).astype(np.int32)
    k_new, v_new = (torch.randn((sum(t), 2, 64), generator=pages.generator).to(DTYPES[dtype]) for _ in range(2))
    K, V, table = pages.to("K", "V", "table")
    positions = torch.full((3, 2, 64), -9, dtype=torch.int32)
    pos = positions.to(gpu_device)
    seen = torch.tensor([1000, 2000, 3000], dtype=torch.int32)
    span.paged_append(k_new.to(gpu_device), v_new.to(gpu_device), K, V, table, torch.tensor(ctx, dtype=torch.int32, device=gpu_device),
                      None if new is None else torch.from_numpy(off).to(gpu_device), positions=pos, seen=seen.to(gpu_device))
    for b in range(3):
        for j in range(t[b]):
            p = ctx[b] - t[b] + j
            if 0 <= p < 64:
                pages.K[pages.table[b, p // 16], :, p % 16], pages.V[pages.table[b, p // 16], :, p % 16] = k_new[off[b] + j], v_new[off[b] + j]
                positions[b, :, p] = int(seen[b]) - t[b] + j
    assert same(K.cpu(), pages.K) and same(V.cpu(), pages.V) and torch.equal(pos.cpu(), positions)


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (3, 1), (10, 0), (40, 5), (64, 2), (70, 0), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_tokens_past_the_table(window, sinks, gpu_device):
    """A chunk whose last tokens have no row: every token sees of the table's positions what it would see of a longer one.  A one-token call is the last of them."""
    cap = 64
    pages = Pages([cap] * 5, 4, 2, 64, 16, "f32", gpu_device, seed=8)
    ctx, new = [66, 64, 90, 200, 2 ** 31 - 1], [5, 3, 40, 1, 4]
    off = np.cumsum([0] + new).astype(np.int32)
    q = torch.randn((sum(new), 4, 64), generator=pages.generator)
    K, V, table = pages.to("K", "V", "table")
    on_gpu = lambda x: torch.as_tensor(x, dtype=torch.int32).to(gpu_device)  # noqa: E731
    got = span.paged_prompt_attn(q.to(gpu_device), K, V, table, on_gpu(ctx), on_gpu(off), 0.125, window=window, sinks=sinks).cpu().double()
    last = q[[int(o) - 1 for o in off[1:]]].contiguous().to(gpu_device)
    weights = torch.zeros((5, 2, cap), device=gpu_device)
    one = span.paged_decode_attn(last, K, V, table, on_gpu(ctx), 0.125, window=window, sinks=sinks, weights=weights).cpu().double()
    sums = torch.zeros((5, 2, cap), dtype=torch.float64)
    for b in range(5):
        for j in range(new[b]):
            at = ctx[b] - new[b] + j
            see = [p for p in range(cap) if p <= at and (window == 0 or p > at - window or p < sinks)]
            out, w = attend(pages, pages.K, pages.V, b, q[off[b] + j], see, 0.125)
            assert float((got[off[b] + j] - out).abs().max()) <= TOL, (b, j)
            if j == new[b] - 1:
                assert float((one[b] - out).abs().max()) <= TOL, b
                sums[b][:, see] = w
    assert float((weights.cpu().double() - sums).abs().max()) <= 2 * TOL  # two heads' weights


def test_a_cache_that_fills_up(gpu_device):
    """Together, from a captured graph: tokens go in until the table is full and past it; what is held stays as it was when the last row fitted."""
    pages = Pages([60], 2, 1, 64, 16, "f16", gpu_device, seed=5, table_pages=4)
    K, V, table, ctx = pages.to("K", "V", "table", "ctx")
    k_new, v_new, q = (torch.zeros((1, n, 64), dtype=torch.float16, device=gpu_device) for n in (1, 1, 2))
    side = torch.cuda.Stream(device=gpu_device)
    append = span.prepare_paged_append(k_new, v_new, K, V, table, ctx, stream=side.cuda_stream)
    look = span.prepare_paged_decode_attn(q, K, V, table, ctx, 0.125, window=20, sinks=2, stream=side.cuda_stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ctx.add_(1)
        append()
        look()
    for n in range(61, 70):
        rows = [torch.randn(x.shape, generator=pages.generator).half() for x in (k_new, v_new, q)]
        for x, y in zip((k_new, v_new, q), rows):
            x.copy_(y)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        if n <= 64:
            pages.K[pages.table[0, 3], :, (n - 1) % 16], pages.V[pages.table[0, 3], :, (n - 1) % 16] = rows[0][0], rows[1][0]
        assert same(K.cpu(), pages.K) and same(V.cpu(), pages.V)
        see = [p for p in range(min(n, 64)) if p >= n - 20 or p < 2]
        assert float((look.out[0].cpu().double() - attend(pages, pages.K, pages.V, 0, rows[2][0], see, 0.125)[0]).abs().max()) <= TOL
