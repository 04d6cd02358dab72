"""One-token attention over pages of 4-bit values in windows that are cut into slices: every output is written and right, and the workspace's counters are zero again."""
import numpy as np
import pytest
import torch

import paper_2404_09336_amd as span
from paged_reference import seen_positions
from paper_2404_09336_amd import paged
from test_gpu_paged_fp4_attn import Fp4Pages, check

pytestmark = pytest.mark.gpu

WINDOWS = [(1536, 0), (1532, 4), (2048, 0), (4096, 0), (4090, 17), (1025, 64)]


class Windowed:
    """A windowed call on a workspace of exactly the bytes that it asks for, its lengths and output the test's."""

    def __init__(self, pages, scale, window, sinks, device):
        self.pages, self.scale, self.window, self.sinks = pages, scale, window, sinks
        B, H, D = len(pages.lens), pages.heads, pages.head_dim
        self.ctx, self.out = torch.zeros(B, dtype=torch.int32, device=device), torch.empty((B, H, D), device=device)
        args = (pages.q.to(device), *pages.cache(), self.ctx, scale, self.out)
        asked = span.paged_workspace_bytes(span.prepare_paged_decode_attn_fp4(*args, window=window, sinks=sinks).desc, paged.PAGED_DECODE_FP4)
        assert asked > 0  # (cut)
        self.workspace = torch.empty(asked, dtype=torch.uint8, device=device)
        self.call = span.prepare_paged_decode_attn_fp4(*args, window=window, sinks=sinks, workspace=self.workspace)
        span.paged_workspace_init(self.call.desc)

    def __call__(self, lens):
        self.ctx.copy_(torch.tensor(lens, dtype=torch.int32))
        self.out.fill_(float("nan"))
        self.call()
        assert not self.workspace[:4 * len(lens) * (self.pages.kv_heads + 1)].any(), lens
        for b, n in enumerate(lens):
            check(self.pages, self.out, b, [p for p in seen_positions(n, self.window, self.sinks) if p < self.pages.capacity], self.scale)


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("heads,kv_heads,head_dim,dtype", [(32, 8, 128, "bf16"), (4, 4, 64, "f32"), (16, 2, 64, "f16"), (7, 1, 128, "f32"), (16, 1, 128, "f16")])
def test_every_remainder_of_a_length(window, sinks, heads, kv_heads, head_dim, dtype, gpu_device):
    """One sequence: windows that begin on a unit and at each of its rows, one call after the other on one workspace; then lengths that the window covers."""
    pages = Fp4Pages([window + 100 + 15], heads, kv_heads, head_dim, 16, dtype, gpu_device, seed=window)
    call = Windowed(pages, head_dim ** -0.5, window, sinks, gpu_device)
    for n in [window + 100 + r for r in range(16)] + [window + r for r in (-1, 0, 1, 7, 16, 17)] + [1, 0, 1500 if window >= 1500 else 900]:
        call([n])


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("batch,heads,kv_heads,page", [(4, 32, 8, 64), (7, 5, 5, 32), (16, 4, 1, 256), (16, 6, 2, 16), (65, 8, 1, 64)])
def test_batches(window, sinks, batch, heads, kv_heads, page, gpu_device):
    """Sequences whose windows begin at different rows of a unit, all at the same, and of very different length."""
    rng = np.random.default_rng(window + batch)
    most = window + 3 * page
    pages = Fp4Pages([most] * batch, heads, kv_heads, 64, page, "bf16", gpu_device, seed=batch)
    call = Windowed(pages, 0.125, window, sinks, gpu_device)
    for lens in ([most - 1] * batch, [most - b % 16 for b in range(batch)], [most] * batch, rng.integers(0, most + 1, batch).tolist(),
                 [most - 5 if b % 3 else int(rng.integers(0, 40)) for b in range(batch)]):
        call(lens)


@pytest.mark.parametrize("over", [0, 1, 9, 300])
def test_tables_that_end_inside_the_window(over, gpu_device):
    """Sinks and window meet in a unit that counts twice; positions past the table are nobody's, and the window goes by the token's own."""
    for window, sinks, table_pages in ((1500, 17, 96), (2048, 33, 128), (2000, 40, 128)):
        pages = Fp4Pages([16 * table_pages] * 2, 8, 2, 64, 16, "bf16", gpu_device, table_pages=table_pages, seed=over)
        call = Windowed(pages, 0.125, window, sinks, gpu_device)
        for off in (0, 1, 15):
            call([16 * table_pages + over + off, max(window + sinks + off, 0)])


def test_replays_as_lengths_grow(gpu_device):
    """A captured step, its length one more each time: the slices follow it."""
    window = 2048
    pages = Fp4Pages([window + 80], 32, 8, 128, 16, "bf16", gpu_device, seed=3)
    call = Windowed(pages, 128 ** -0.5, window, 0, gpu_device)
    side = torch.cuda.Stream(device=gpu_device)
    grown = span.prepare_paged_decode_attn_fp4(pages.q.to(gpu_device), *pages.cache(), call.ctx, call.scale, call.out, window=window, workspace=call.workspace,
                                               stream=side.cuda_stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call.ctx.add_(1)
        grown()
    call.ctx.fill_(window + 40)
    for n in range(window + 41, window + 41 + 35):
        call.out.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert not call.workspace[:4 * 9].any()
        check(pages, call.out, 0, range(n - window, n), call.scale)
