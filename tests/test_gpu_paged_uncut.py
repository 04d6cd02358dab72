"""One-token calls whose batch alone fills the card: no sequence is cut whatever the lengths, and where they are short the workgroup that attends adds up the weights."""
import numpy as np
import pytest
import torch

import paper_2404_09336_amd as span
from paged_reference import Pages, attend, seen_positions

pytestmark = pytest.mark.gpu
TOL = 1e-5


@pytest.mark.parametrize("dtype,head_dim", [("f32", 64), ("f16", 128), ("bf16", 64)])
@pytest.mark.parametrize("heads,kv_heads,batch", [(64, 32, 33), (128, 128, 8), (16, 8, 128), (32, 32, 32)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 4)])
def test_batches_that_are_never_cut(dtype, head_dim, heads, kv_heads, batch, window, sinks, gpu_device):
    """Empty, short and long sequences side by side, with weights and without; from a graph as well, replayed while the lengths change."""
    rng = np.random.default_rng(batch)
    lens = [int(n) for n in rng.integers(0, 120, batch)]
    lens[1], lens[2], lens[-1] = 900 if batch != 32 else 2600, 0, 610  # (32 x 32 x 2600: too many for the workgroups' own pass)
    pages = Pages(lens, heads, kv_heads, head_dim, 32, dtype, gpu_device, seed=batch)
    q, K, V, table, ctx = pages.to("q", "K", "V", "table", "ctx")
    side = torch.cuda.Stream(device=gpu_device)
    weights = torch.zeros((batch, kv_heads, pages.capacity), device=gpu_device)
    kw = dict(window=window, sinks=sinks)
    call = span.prepare_paged_decode_attn(q, K, V, table, ctx, head_dim ** -0.5, weights=weights, stream=side.cuda_stream, **kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for now in (lens, [n // 2 for n in lens], lens):
        ctx.copy_(torch.tensor(now, dtype=torch.int32))
        weights.fill_(0.5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got, sums = call.out.cpu().double(), weights.cpu().double()
        plain = span.paged_decode_attn(q, K, V, table, ctx, head_dim ** -0.5, **kw)
        assert torch.equal(plain, call.out)
        for b in range(batch):
            see = seen_positions(now[b], window, sinks)
            out, w = attend(pages, pages.K, pages.V, b, pages.q[b], see, head_dim ** -0.5)
            assert float((got[b] - out).abs().max()) <= TOL, b
            want = torch.full((kv_heads, pages.capacity), 0.5, dtype=torch.float64)
            want[:, see] += w
            assert float((sums[b] - want).abs().max()) <= 2 * TOL  # two heads' weights at most
