"""Attention of new tokens over a cache in pages against the 64-bit form: ragged chunks, windows and sinks, what lies in masked places."""
import numpy as np
import pytest
import torch

import paper_2404_09336_amd as span
from paged_reference import DTYPES, Pages

pytestmark = pytest.mark.gpu
# Scores of N(0, 1) rows scaled by head_dim^-0.5 are off by some 1e-6 and so are fp32 weights and outputs: 1e-5, as for the one-token calls.  With 16
# bits a weight w_j is rounded to half a step of its type (eps / 2 relative), and so is the output: at most eps / 2 * (sum_j w_j |v_j| + |out|).
STEP = {"f32": 0.0, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


class Prompt(Pages):
    def __init__(self, lens, new, heads, kv_heads, head_dim, page, dtype, device, seed=0, **kw):
        super().__init__(lens, heads, kv_heads, head_dim, page, dtype, device, seed=seed, **kw)
        self.new, self.dtype = list(new), dtype
        self.off = torch.from_numpy(np.cumsum([0] + self.new).astype(np.int32))
        self.q = torch.randn((sum(self.new), heads, head_dim), generator=self.generator).to(DTYPES[dtype])

    def reference(self, window=0, sinks=0, scale=None, missing=()):
        """(out, allowed error), both [tokens, heads, head_dim] in 64 bits.  missing: (sequence, page of it) that nobody attends."""
        scale = self.head_dim ** -0.5 if scale is None else scale
        G = self.heads // self.kv_heads
        out, err = (torch.zeros(self.q.shape, dtype=torch.float64) for _ in range(2))
        for b, (n, t) in enumerate(zip(self.lens, self.new)):
            if t == 0 or n == 0:
                continue
            first = int(self.off[b])
            at = torch.arange(n - t, n)[:, None]
            p = torch.arange(n)
            sees = (p <= at) & ((p > at - window) | (p < sinks) if window else True)
            for mb, page in missing:
                if mb == b:
                    sees = sees & (p // self.page != page)
            k, v = (self.rows(pool, b, range(n)) for pool in (self.K, self.V))
            for i in range(self.heads):
                s = self.q[first:first + t, i].double() @ k[i // G].T.contiguous() * scale
                s = torch.where(sees, s, torch.tensor(-np.inf, dtype=torch.float64))
                w = torch.softmax(s, -1)
                w = torch.where(sees, w, torch.zeros_like(w))
                w[~sees.any(-1)] = 0
                vi = v[i // G]
                masked = torch.where(torch.isfinite(vi), vi, torch.zeros_like(vi))
                o = w @ masked
                wild = (~torch.isfinite(vi)).any(-1).nonzero().flatten().tolist()
                for j in wild:  # only tokens that see the row meet it
                    row = torch.where(torch.isfinite(vi[j]), torch.zeros_like(vi[j]), vi[j])
                    o += torch.where(sees[:, j, None] & (row != 0), w[:, j, None] * row, torch.zeros_like(o))
                out[first:first + t, i] = o
                err[first:first + t, i] = STEP[self.dtype] * (w @ masked.abs() + o.abs())
        return out, err + 1e-5

    def check(self, window=0, sinks=0, scale=None, missing=(), **kw):
        q, K, V, table, ctx, off = self.to("q", "K", "V", "table", "ctx", "off")
        got = span.paged_prompt_attn(q, K, V, table, ctx, off, self.head_dim ** -0.5 if scale is None else scale, window=window, sinks=sinks, **kw)
        assert got.dtype == q.dtype
        got = got.cpu().double()
        want, err = self.reference(window, sinks, scale, missing)
        odd = ~torch.isfinite(want)
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[odd & ~torch.isnan(want)], want[odd & ~torch.isnan(want)])
        off_by = (got - want).abs()[~odd] - err[~odd]
        assert off_by.numel() == 0 or float(off_by.max()) <= 0
        return got


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (4, 4), (8, 2), (7, 1), (16, 1), (15, 3)])
def test_lengths_and_groups(dtype, head_dim, heads, kv_heads, gpu_device):
    """Chunks of 0 to 300 tokens behind 0 to 600 cached ones; more new tokens than positions; no positions at all."""
    Prompt([1, 17, 64, 65, 300, 700, 5, 0, 130], [1, 3, 64, 1, 300, 100, 9, 2, 0], heads, kv_heads, head_dim, 16, dtype, gpu_device, seed=heads).check()


@pytest.mark.parametrize("dtype,head_dim", [("f32", 64), ("f16", 128), ("bf16", 64)])
@pytest.mark.parametrize("page", [16, 32, 64, 256, 1024])
def test_pages(dtype, head_dim, page, gpu_device):
    Prompt([1500, 77, 513], [600, 77, 129], 4, 2, head_dim, page, dtype, gpu_device, seed=page).check()


@pytest.mark.parametrize("dtype,head_dim", [("f32", 128), ("f16", 64), ("bf16", 128)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (16, 16), (63, 64), (64, 65), (100, 4), (129, 200), (1000, 1), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_window_and_sinks(dtype, head_dim, window, sinks, gpu_device):
    Prompt([1, 400, 640, 90], [1, 400, 300, 30], 6, 2, head_dim, 32, dtype, gpu_device, seed=window % 97).check(window, sinks)


@pytest.mark.parametrize("heads,kv_heads", [(32, 8), (8, 8), (40, 5)])
def test_many_tiles(heads, kv_heads, gpu_device):
    """Enough tiles that no two workgroups share one."""
    p = Prompt([900, 1024, 33], [900, 700, 33], heads, kv_heads, 128, 64, "bf16", gpu_device, seed=heads)
    p.check()
    p.check(window=200, sinks=4)


@pytest.mark.parametrize("batch", [64, 65, 200])
def test_many_sequences(batch, gpu_device):
    rng = np.random.default_rng(batch)
    new = [int(n) for n in rng.integers(0, 12, batch) * (rng.random(batch) < 0.7)]
    new[-1] = 40
    Prompt([n + int(c) for n, c in zip(new, rng.integers(0, 60, batch))], new, 4, 1, 64, 16, "f16", gpu_device, seed=batch).check()


@pytest.mark.parametrize("dtype,head_dim", [("f32", 64), ("f16", 128), ("bf16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("few", [False, True])
def test_rows_that_are_not_finite_in_masked_places(dtype, head_dim, few, gpu_device):
    """NaN and Inf in K and V rows of later positions, before a window, and past the length (there Pages puts NaN): tokens that do not see them are
    not touched by them; tokens that do have exactly the elements that the definition has."""
    lens, new = ([200, 150], [200, 60]) if few else ([700, 900, 650], [700, 600, 650])
    p = Prompt(lens, new, 32 if not few else 2, 8 if not few else 1, head_dim, 32, dtype, gpu_device, seed=21)
    row = lambda b, i: (p.table[b, i // 32], slice(None), i % 32)  # noqa: E731
    p.V[row(0, 120)][..., 5] = float("inf")
    p.V[row(0, 121)][..., head_dim - 1] = float("-inf")
    p.V[row(0, 199)][..., 7] = float("nan")
    p.V[row(1, 140)] = float("nan")
    p.K[row(1, 149)] = float("nan")
    p.check()
    p.check(window=20, sinks=2)


def test_pages_outside_the_pool(gpu_device):
    p = Prompt([400, 90], [150, 90], 8, 4, 128, 16, "f16", gpu_device, seed=5, table_pages=40)
    missing = [(0, 0), (0, 7), (0, 20), (1, 5)]
    for k, (b, i) in enumerate(missing):
        p.table[b, i] = [-1, p.K.shape[0], 2 ** 31 - 1, -2 ** 31][k]
    p.table[:, 30:] = -7
    p.check(missing=missing)


@pytest.mark.parametrize("scale", [2.0 ** 20, -0.3, 0.0])
def test_scales(scale, gpu_device):
    """Scaled scores of 2^20 (one row has all the weight), a negative scale, zero."""
    for dtype in ("f32", "f16", "bf16"):
        Prompt([100], [100], 2, 1, 64, 16, dtype, gpu_device, seed=2).check(scale=scale)


def test_rows_of_nobody_stay(gpu_device):
    """Rows of out that no sequence has; offsets that leave gaps at both ends."""
    p = Prompt([50, 20], [30, 20], 4, 2, 64, 16, "bf16", gpu_device, seed=1)
    q, K, V, table, ctx, off = p.to("q", "K", "V", "table", "ctx", "off")
    wide = torch.cat([q.new_full((3, 4, 64), float("nan")), q, q.new_full((5, 4, 64), float("nan"))])
    out = torch.full_like(wide, 7.0)
    span.paged_prompt_attn(wide, K, V, table, ctx, off + 3, 0.125, out)
    assert (out[:3] == 7).all() and (out[53:] == 7).all()
    assert torch.equal(out[3:53], span.paged_prompt_attn(q, K, V, table, ctx, off, 0.125))


def test_one_token_is_the_one_token_call(gpu_device):
    p = Prompt([700, 33, 1, 2000], [1, 1, 1, 1], 8, 2, 128, 16, "f32", gpu_device, seed=3)
    q, K, V, table, ctx, off = p.to("q", "K", "V", "table", "ctx", "off")
    for window, sinks in ((0, 0), (100, 4)):
        a = span.paged_prompt_attn(q, K, V, table, ctx, off, 128 ** -0.5, window=window, sinks=sinks)
        b = span.paged_decode_attn(q, K, V, table, ctx, 128 ** -0.5, window=window, sinks=sinks)
        assert float((a - b).abs().max()) <= 2e-5


def test_a_prompt_in_chunks_then_tokens(gpu_device):
    """As a program uses them: a prompt goes in chunk by chunk (append, attend), every chunk's outputs are those of the prompt at once."""
    H, KV, D, P, n = 8, 2, 128, 16, 500
    g = torch.Generator(device=gpu_device).manual_seed(3)
    k, v, q = (torch.randn((n, h, D), device=gpu_device, generator=g).bfloat16() for h in (KV, KV, H))
    K, V = (torch.zeros((40, KV, P, D), dtype=torch.bfloat16, device=gpu_device) for _ in range(2))
    table = torch.randperm(40, device=gpu_device, generator=g).to(torch.int32)[None, :32].contiguous()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=gpu_device)  # noqa: E731
    outs, at = [], 0
    for t in (1, 128, 200, 7, 163, 1):
        rows = slice(at, at + t)
        at += t
        span.paged_append(k[rows], v[rows], K, V, table, i32(at), i32(0, t))
        outs.append(span.paged_prompt_attn(q[rows], K, V, table, i32(at), i32(0, t), D ** -0.5))
    whole = span.paged_prompt_attn(q, K, V, table, i32(n), i32(0, n), D ** -0.5)
    err = (torch.cat(outs).double() - whole.double()).abs()
    assert float((err - 2.0 ** -7 * whole.double().abs()).max()) <= 2.0 ** -7  # both sides round weights (of sum 1, |v| < 5) and outputs


def test_graph_follows_the_lengths(gpu_device):
    """A captured call, with and without shared tiles, replayed while lengths, offsets and tables change."""
    for heads, kv in ((8, 2), (64, 16)):
        p = Prompt([700, 300, 90], [200, 300, 40], heads, kv, 128, 16, "f16", gpu_device, seed=heads)
        q, K, V, table, ctx, off = p.to("q", "K", "V", "table", "ctx", "off")
        side = torch.cuda.Stream(device=gpu_device)
        call = span.prepare_paged_prompt_attn(q, K, V, table, ctx, off, 128 ** -0.5, window=150, sinks=4, stream=side.cuda_stream)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
        for lens, offs in (([700, 300, 90], [0, 200, 500, 540]), ([40, 290, 90], [0, 40, 300, 390]), ([700, 300, 90], [0, 0, 300, 300])):
            ctx.copy_(torch.tensor(lens, dtype=torch.int32))
            off.copy_(torch.tensor(offs, dtype=torch.int32))
            call.out.zero_()
            torch.randn(1 << 20, device=gpu_device).sum()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            eager = span.paged_prompt_attn(q, K, V, table, ctx, off, 128 ** -0.5, torch.zeros_like(q), window=150, sinks=4)
            torch.cuda.synchronize()
            assert torch.equal(call.out, eager)
