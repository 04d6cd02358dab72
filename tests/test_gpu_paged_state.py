"""What calls on a cache in pages leave behind: the workspace's counters, entries of weights that nobody attended, the cache itself."""
import pytest
import torch

import paper_2404_09336_amd as span
from paged_reference import Pages, seen_positions

pytestmark = pytest.mark.gpu


def bits(t):
    return t.contiguous().view(torch.uint8)


@pytest.mark.parametrize("spans,window,sinks", [(False, 0, 0), (False, 700, 4), (True, 0, 0)])
@pytest.mark.parametrize("num_splits", [0, 1, 5])
def test_one_token_calls_leave_their_surroundings(spans, window, sinks, num_splits, gpu_device):
    """Sliced and whole calls with weights on the caller's workspace, again and again: the counters are zero after each, and its bytes past them that the call did not ask
    for are as they were; weights of positions that no token sees, K and V keep their bits; outputs are the same every time."""
    lens = [3000, 50, 1234, 0, 300]
    pages = Pages(lens, 8, 2, 128, 16, "bf16", gpu_device, seed=8, table_pages=200)
    q, K, V, table, ctx = pages.to("q", "K", "V", "table", "ctx")
    K0, V0 = K.clone(), V.clone()
    lists = [[(0, n)] if n else [] for n in lens]
    if spans:
        lists[0] = [(5, 2000), (2100, 2999)]
        off = torch.tensor([0] + [len(x) for x in lists]).cumsum(0).to(torch.int32).to(gpu_device)
        st, en = (torch.tensor([iv[k] for x in lists for iv in x], dtype=torch.int32, device=gpu_device) for k in (0, 1))
        see = [[p for s, e in x for p in range(s, e)] for x in lists]
    else:
        see = [seen_positions(n, window, sinks) for n in lens]
    room = 1 << 23
    workspace = torch.full((room,), 0x5a, dtype=torch.uint8, device=gpu_device)
    weights = torch.rand((5, 2, pages.capacity), device=gpu_device) - 0.5
    start = weights.clone()
    kw = dict(weights=weights, num_splits=num_splits, workspace=workspace)
    if spans:
        call = span.prepare_paged_span_decode_attn(q, K, V, table, off, st, en, 128 ** -0.5, **kw)
    else:
        call = span.prepare_paged_decode_attn(q, K, V, table, ctx, 128 ** -0.5, window=window, sinks=sinks, **kw)
    asked = span.paged_workspace_bytes(call.desc, 3 if spans else 1)
    counters = -(-4 * 5 * (2 + 1) // 256) * 256
    assert counters < asked < room
    span.paged_workspace_init(call.desc)
    first = None
    for _ in range(10):
        out = call().clone()
        first = out if first is None else first
        torch.cuda.synchronize()
        assert torch.equal(out, first)
        assert not workspace[:counters].any() and (workspace[asked:] == 0x5a).all()
    seen = torch.zeros((5, pages.capacity), dtype=torch.bool)
    for b, p in enumerate(see):
        seen[b, p] = True
    unseen = ~seen[:, None].expand(5, 2, -1).to(gpu_device)
    assert torch.equal(weights[unseen], start[unseen]) and not torch.equal(weights, start)
    assert torch.equal(bits(K), bits(K0)) and torch.equal(bits(V), bits(V0))
