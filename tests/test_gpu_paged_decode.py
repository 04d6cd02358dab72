"""One-token attention over a cache in pages against the 64-bit form: shapes, slices, windows, span lists, weights per position, and what
rows outside the attended ones hold."""
import numpy as np
import pytest
import torch

import paper_2404_09336_amd as span
from paged_reference import Pages, attend, seen_positions

pytestmark = pytest.mark.gpu
# As for the contiguous cache (test_gpu_matrix): a score of N(0, 1) rows scaled by head_dim^-0.5 is a sum of 128 products at most, off by some
# 1e-6; weights and outputs of size 1 then by a few 1e-6 at most, ten times what the sums' rounding adds up to in practice.
TOL = 1e-5


def check(pages, positions_of, call, K=None, V=None, weights=None, tol=TOL):
    """`call` gives out; positions_of(b) the attended positions.  weights: (before, after) or None."""
    K, V = pages.K if K is None else K, pages.V if V is None else V
    got = call().cpu().double()
    want_w = None if weights is None else weights[0].cpu().double().clone()
    for b in range(len(pages.lens)):
        p = positions_of(b)
        out, w = attend(pages, K, V, b, pages.q[b], p, pages.head_dim ** -0.5)
        assert float((got[b] - out).abs().max()) <= tol, (b, pages.lens[b])
        if want_w is not None:
            want_w[b][:, torch.as_tensor(np.asarray(p, dtype=np.int64))] += w
    if weights is not None:
        # a sum of up to 16 weights of at most 1, each off by its score's error, and the addition's rounding
        assert float((weights[1].cpu().double() - want_w).abs().max()) <= 16 * tol


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (4, 4), (8, 2), (7, 1), (16, 1), (15, 3)])
def test_lengths_and_groups(dtype, head_dim, heads, kv_heads, gpu_device):
    """Lengths around tiles, pages and slices; an empty sequence; a group of 1 to 16 heads."""
    pages = Pages([1, 2, 15, 16, 17, 0, 31, 33, 64, 127, 128, 129, 300, 1000], heads, kv_heads, head_dim, 16, dtype, gpu_device, seed=heads)
    q, K, V, table, ctx = pages.to("q", "K", "V", "table", "ctx")
    check(pages, lambda b: range(pages.lens[b]), lambda: span.paged_decode_attn(q, K, V, table, ctx, head_dim ** -0.5))


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256, 512, 1024])
@pytest.mark.parametrize("num_splits", [0, 1, 3, 40])
def test_pages_and_slices(page, num_splits, gpu_device):
    pages = Pages([1500, 1, 777, 2049], 8, 2, 128, page, "bf16", gpu_device, seed=page)
    q, K, V, table, ctx = pages.to("q", "K", "V", "table", "ctx")
    check(pages, lambda b: range(pages.lens[b]), lambda: span.paged_decode_attn(q, K, V, table, ctx, 128 ** -0.5, num_splits=num_splits))


@pytest.mark.parametrize("batch", [1, 3, 63, 64, 65, 130, 520])
def test_slices_found_on_the_device(batch, gpu_device):
    """Ragged batches on both sides of a wave's 64 sequences and of the largest batch that is sliced by its lengths."""
    rng = np.random.default_rng(batch)
    lens = [int(n) for n in rng.integers(0, 400, batch)]
    lens[-1] = 1700
    pages = Pages(lens, 2, 1, 64, 64, "f16", gpu_device, seed=batch)
    q, K, V, table, ctx = pages.to("q", "K", "V", "table", "ctx")
    check(pages, lambda b: range(lens[b]), lambda: span.paged_decode_attn(q, K, V, table, ctx, 0.125))


@pytest.mark.parametrize("dtype,head_dim", [("f32", 128), ("f16", 64), ("bf16", 128)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (16, 16), (100, 4), (129, 200), (1000, 1), (5000, 64), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("with_weights", [False, True])
def test_window_and_sinks(dtype, head_dim, window, sinks, with_weights, gpu_device):
    """The rows between the sinks and the window hold NaN: nobody reads them."""
    pages = Pages([0, 1, 4, 99, 100, 101, 130, 700, 1100], 4, 2, head_dim, 32, dtype, gpu_device, seed=3)
    see = [seen_positions(n, window, sinks) for n in pages.lens]
    for b, n in enumerate(pages.lens):
        for p in set(range(n)) - set(see[b]):
            pages.K[pages.table[b, p // 32], :, p % 32] = float("nan")
            pages.V[pages.table[b, p // 32], :, p % 32] = float("inf")
    q, K, V, table, ctx = pages.to("q", "K", "V", "table", "ctx")
    before = torch.rand((len(pages.lens), 2, pages.capacity), device=gpu_device)
    after = before.clone()
    kw = {"weights": after} if with_weights else {}
    check(pages, lambda b: see[b], lambda: span.paged_decode_attn(q, K, V, table, ctx, head_dim ** -0.5, window=window, sinks=sinks, **kw),
          weights=(before, after) if with_weights else None)


def lists(rng, n, count):
    """Disjoint intervals of [0, n) in any order."""
    cuts = np.sort(rng.choice(n + 1, 2 * count, replace=False))
    iv = [(int(a), int(b)) for a, b in zip(cuts[::2], cuts[1::2])]
    rng.shuffle(iv)
    return iv


@pytest.mark.parametrize("dtype,head_dim", [("f32", 64), ("f16", 128), ("bf16", 64)])
@pytest.mark.parametrize("counts", ["none", "true", "wrong"])
@pytest.mark.parametrize("with_weights", [False, True])
def test_spans(dtype, head_dim, counts, with_weights, gpu_device):
    """1 to 150 intervals of a sequence, an empty list, one position, the whole cache; host counts that are right, wrong or not there."""
    rng = np.random.default_rng(7)
    lens = [50, 2000, 900, 1, 640, 3000, 17]
    iv = [lists(rng, 50, 3), lists(rng, 2000, 20), [], [(0, 1)], [(0, 640)], lists(rng, 3000, 150), [(3, 4), (16, 17)]]
    pages = Pages(lens, 6, 3, head_dim, 16, dtype, gpu_device, seed=11)
    off = np.cumsum([0] + [len(x) for x in iv]).astype(np.int32)
    st, en = (np.array([x[k] for seq in iv for x in seq], np.int32) for k in (0, 1))
    see = [[p for s, e in seq for p in range(s, e)] for seq in iv]
    tokens = {"none": None, "true": [len(s) for s in see], "wrong": [1, 5000, 0, 700, 3, 3, 10 ** 9]}[counts]
    q, K, V, table = pages.to("q", "K", "V", "table")
    dev = [torch.from_numpy(a).to(gpu_device) for a in (off, st, en)]
    before = torch.rand((len(lens), 3, pages.capacity), device=gpu_device)
    after = before.clone()
    check(pages, lambda b: see[b], lambda: span.paged_span_decode_attn(q, K, V, table, *dev, head_dim ** -0.5, tokens_per_seq=tokens,
                                                                       weights=after if with_weights else None),
          weights=(before, after) if with_weights else None)


def test_span_form_equals_the_contiguous_cache(gpu_device):
    """A sequence whose pages follow one another is a contiguous cache: span_decode_attn gives the same to rounding."""
    B, H, L, D = 3, 4, 512, 128
    g = torch.Generator(device=gpu_device).manual_seed(1)
    K, V = (torch.randn((B, H, L, D), device=gpu_device, generator=g).half() for _ in range(2))
    q = torch.randn((B, H, D), device=gpu_device, generator=g).half()
    off, st, en = (torch.tensor(x, dtype=torch.int32, device=gpu_device) for x in ([0, 2, 3, 5], [0, 100, 7, 0, 500], [30, 350, 480, 1, 512]))
    want = span.span_decode_attn(q, K, V, off, st, en, None, D ** -0.5)
    table = torch.arange(B, dtype=torch.int32, device=gpu_device)[:, None].contiguous()
    got = span.paged_span_decode_attn(q, K, V, table, off, st, en, D ** -0.5)
    assert float((got - want).abs().max()) <= 2 * TOL


def test_pages_outside_the_pool_and_long_tables(gpu_device):
    """Positions of such pages are attended by nobody, weights there stay as they are; a table may be longer than any sequence."""
    pages = Pages([400, 90, 33], 8, 4, 128, 16, "f16", gpu_device, seed=5, table_pages=40)
    bad = {0: [0, 7, 24], 1: [5], 2: [0, 1, 2]}
    table = pages.table.clone()
    for b, entries in bad.items():
        for k, i in enumerate(entries):
            table[b, i] = [-1, pages.K.shape[0], 2 ** 31 - 1][k % 3]
    table[:, 30:] = -7
    see = [[p for p in range(n) if p // 16 not in bad[b]] for b, n in enumerate(pages.lens)]
    q, K, V, ctx = pages.to("q", "K", "V", "ctx")
    before = torch.rand((3, 4, pages.capacity), device=gpu_device)
    after = before.clone()
    check(pages, lambda b: see[b], lambda: span.paged_decode_attn(q, K, V, table.to(gpu_device), ctx, 128 ** -0.5, weights=after), weights=(before, after))


def test_lengths_are_clamped(gpu_device):
    pages = Pages([64, 64], 2, 2, 64, 16, "f32", gpu_device)
    q, K, V, table = pages.to("q", "K", "V", "table")
    ctx = torch.tensor([2 ** 31 - 1, -5], dtype=torch.int32, device=gpu_device)
    got = span.paged_decode_attn(q, K, V, table, ctx, 0.125).cpu().double()
    assert float((got[0] - attend(pages, pages.K, pages.V, 0, pages.q[0], range(64), 0.125)[0]).abs().max()) <= TOL
    assert not got[1].any()


@pytest.mark.parametrize("num_splits", [1, 5])
def test_scores_that_are_not_finite(num_splits, gpu_device):
    """An attended K row with NaN or an overflowing score makes the rows of its heads NaN, one of -Inf has no weight."""
    pages = Pages([520, 520, 520, 520], 4, 2, 128, 64, "f16", gpu_device, seed=9)
    row = lambda b, p: (pages.table[b, p // 64], slice(None), p % 64)  # noqa: E731
    pages.K[row(0, 203)] = float("nan")
    sign = torch.where(pages.q[1, ::2] >= 0, float("inf"), float("-inf")).half()
    pages.K[row(1, 7)] = sign                        # the first head of each group sees +Inf
    pages.q[1, 1::2] = pages.q[1, ::2]               # and so does the second
    pages.q[2, 1::2] = pages.q[2, ::2]
    pages.K[row(2, 519)] = torch.where(pages.q[2, ::2] >= 0, float("-inf"), float("inf")).half()
    q, K, V, table, ctx = pages.to("q", "K", "V", "table", "ctx")
    got = span.paged_decode_attn(q, K, V, table, ctx, 128 ** -0.5, num_splits=num_splits).cpu().double()
    assert got[0].isnan().all() and got[1].isnan().all() and not got[2:].isnan().any()
    want = attend(pages, pages.K, pages.V, 2, pages.q[2], range(519), 128 ** -0.5)[0]
    assert float((got[2] - want).abs().max()) <= TOL


def test_large_scores(gpu_device):
    """Scaled scores of 2^20: one row takes all the weight, whatever the scores' size."""
    pages = Pages([300], 2, 1, 128, 16, "bf16", gpu_device, seed=2)
    q, K, V, table, ctx = pages.to("q", "K", "V", "table", "ctx")
    got = span.paged_decode_attn(q, K, V, table, ctx, 2.0 ** 20).cpu().double()
    want = attend(pages, pages.K, pages.V, 0, pages.q[0], range(300), 2.0 ** 20)[0]
    assert float((got[0] - want).abs().max()) <= TOL


def test_calls_are_repeatable_and_keep_to_their_own(gpu_device):
    """The same bits call after call on one workspace; the workspace's counters, entries of weights that were not attended and the cache stay."""
    pages = Pages([3000, 50, 1234], 8, 2, 128, 16, "bf16", gpu_device, seed=8, table_pages=200)
    q, K, V, table, ctx = pages.to("q", "K", "V", "table", "ctx")
    K0 = K.clone()
    call = span.prepare_paged_decode_attn(q, K, V, table, ctx, 128 ** -0.5)
    first = call().clone()
    for _ in range(50):
        assert torch.equal(call(), first)
    assert torch.equal(K.view(torch.int16), K0.view(torch.int16))


def test_graph_follows_the_lengths(gpu_device):
    """A captured call with weights, replayed while ctx_lens and the block table change: every replay is the eager result."""
    pages = Pages([1500, 40, 600], 8, 2, 128, 16, "bf16", gpu_device, seed=4)
    q, K, V, table, ctx = pages.to("q", "K", "V", "table", "ctx")
    side = torch.cuda.Stream(device=gpu_device)
    weights = torch.zeros((3, 2, pages.capacity), device=gpu_device)
    call = span.prepare_paged_decode_attn(q, K, V, table, ctx, 128 ** -0.5, weights=weights, stream=side.cuda_stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for lens in ([1500, 40, 600], [1, 0, 599], [900, 39, 3], [1500, 40, 600]):
        ctx.copy_(torch.tensor(lens, dtype=torch.int32))
        weights.zero_()
        torch.randn(1 << 20, device=gpu_device).sum()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        again = torch.zeros_like(weights)
        eager = span.paged_decode_attn(q, K, V, table, ctx, 128 ** -0.5, weights=again)
        torch.cuda.synchronize()
        assert torch.equal(call.out, eager) and torch.equal(weights, again), lens


def test_pools_past_32_bits(gpu_device):
    """A pool of more than 4 GiB whose last pages hold the sequence."""
    N, KV, P, D = 2200, 8, 1024, 128                 # 4.6 GB of K
    K, V = (torch.zeros((N, KV, P, D), dtype=torch.float16, device=gpu_device) for _ in range(2))
    g = torch.Generator(device=gpu_device).manual_seed(3)
    last = [N - 1, N - 2, 3]
    for i in last:
        K[i], V[i] = (torch.randn((KV, P, D), device=gpu_device, generator=g).half() for _ in range(2))
    q = torch.randn((1, 16, D), device=gpu_device, generator=g).half()
    table = torch.tensor([last], dtype=torch.int32, device=gpu_device)
    ctx = torch.tensor([2500], dtype=torch.int32, device=gpu_device)
    got = span.paged_decode_attn(q, K, V, table, ctx, D ** -0.5).cpu().double()
    k, v = (torch.cat([x[i] for i in last], 1)[:, :2500].cpu().double() for x in (K, V))
    w = torch.softmax(torch.matmul(q[0].cpu().double().reshape(KV, 2, D), k.transpose(1, 2).contiguous()) * D ** -0.5, -1)
    assert float((got[0] - torch.matmul(w, v).reshape(16, D)).abs().max()) <= TOL
