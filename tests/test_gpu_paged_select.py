"""Page selection: bounds and lists have to be equal to the 64-bit form's; attention over lists is off by its roundings."""
import numpy as np
import pytest
import torch

import paper_2404_09336_amd as span
from paged_more_reference import select
from paged_reference import DTYPES, Pages, attend

pytestmark = pytest.mark.gpu


def reference_bounds(pages, lens, since, before):
    """What the call leaves in bounds [pages, kv_heads, 2, D]."""
    out = before.clone()
    N = pages.K.shape[0]
    for b, n in enumerate(lens):
        n = min(max(n, 0), pages.capacity)
        for j in range(-(-n // pages.page)):
            first, end = j * pages.page, min((j + 1) * pages.page, n)
            page = int(pages.table[b, j])
            if end <= since[b] or not 0 <= page < N:
                continue
            rows = pages.K[page, :, max(since[b] - first, 0):end - first].float()
            lo, hi = rows.amin(1), rows.amax(1)  # (torch's let NaN through)
            if since[b] > first:
                lo, hi = torch.minimum(lo, before[page, :, 0].float()), torch.maximum(hi, before[page, :, 1].float())
            out[page, :, 0], out[page, :, 1] = lo.to(out.dtype), hi.to(out.dtype)
    return out


def reference_lists(pages, q, bounds, lens, budget, sinks, recent):
    G = pages.heads // pages.kv_heads
    out = []
    for b, n in enumerate(lens):
        n = min(max(n, 0), pages.capacity)
        for h in range(pages.kv_heads):
            out.append(select(q[b, h * G:(h + 1) * G].double().numpy(), bounds[:, h].double().numpy(), n, pages.table[b].tolist(), pages.page, budget, sinks, recent))
    return torch.tensor(out, dtype=torch.int32).reshape(len(lens), pages.kv_heads, budget)


def same(a, b):
    """Equal, NaN to NaN and zeros of either sign to one another."""
    a, b = a.cpu().float(), b.cpu().float()
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(nan=1.5), b.nan_to_num(nan=1.5))


def run(pages, q, bounds, lens, budget, device, **kw):
    K, table = pages.to("K", "table")
    ctx = torch.tensor(lens, dtype=torch.int32, device=device)
    since = kw.pop("since", None)
    b = bounds.to(device)
    got = span.paged_select(q.to(device), K, b, table, ctx, budget, since=None if since is None else torch.tensor(since, dtype=torch.int32, device=device), **kw)
    return got.cpu(), b.cpu()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads,kv_heads,head_dim,page", [(4, 4, 64, 16), (16, 1, 128, 16), (14, 2, 64, 32), (6, 3, 128, 64)])
@pytest.mark.parametrize("budget,sinks,recent", [(4, 0, 0), (7, 16, 20), (12, 1, 17), (40, 0, 1)])
def test_select_after_prompts(dtype, heads, kv_heads, head_dim, page, budget, sinks, recent, gpu_device):
    """All bounds are made; lengths from none to more pages than a workgroup takes, below and above the budget."""
    lens = [0, 1, page, page + 1, 4 * page, 5 * page - 1, 33 * page, 34 * page + 3, 70 * page + 5, 129 * page]
    pages = Pages(lens, heads, kv_heads, head_dim, page, dtype, gpu_device, seed=budget)
    N = pages.K.shape[0]
    bounds = torch.full((N, kv_heads, 2, head_dim), 9.0).to(DTYPES[dtype])
    got, b = run(pages, pages.q, bounds, lens, budget, gpu_device, sinks=sinks, recent=recent, since=[0] * len(lens))
    want = reference_bounds(pages, lens, [0] * len(lens), bounds)
    assert same(b, want)
    assert torch.equal(got, reference_lists(pages, pages.q, want, lens, budget, sinks, recent))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("since", ["none", "some"])
def test_select_step_by_step(dtype, since, gpu_device):
    """New rows join bounds that earlier calls made; a row that begins a page makes them anew."""
    lens = [300, 17, 16, 1, 257, 0]
    pages = Pages(lens, 4, 2, 64, 16, dtype, gpu_device, seed=5, table_pages=20)
    start = [max(n - 1, 0) for n in lens] if since == "none" else [250, 16, 16, 0, 1, 0]
    bounds = torch.full((pages.K.shape[0], 2, 2, 64), 9.0).to(DTYPES[dtype])
    bounds = reference_bounds(pages, start, [0] * 6, bounds)     # of the rows ahead of the new ones
    got, b = run(pages, pages.q, bounds, lens, 5, gpu_device, since=None if since == "none" else start)
    want = reference_bounds(pages, lens, start, bounds)
    assert same(b, want) and torch.equal(got, reference_lists(pages, pages.q, want, lens, 5, 0, 1))
    whole = reference_bounds(pages, lens, [0] * 6, bounds)
    assert same(want, whole)
    # again with the same arguments: nothing changes
    again, b2 = run(pages, pages.q, b, lens, 5, gpu_device, since=None if since == "none" else start)
    assert same(b2, b) and torch.equal(again, got)


def test_ties_go_to_the_lower_page(gpu_device):
    """Pages of equal rows; two levels of them, the border in the middle of one; zeros of either sign are equal."""
    lens = [40 * 16]
    pages = Pages(lens, 2, 1, 64, 16, "f32", gpu_device)
    level = torch.tensor([1.0, 2.0, 2.0, 3.0] * 10)
    for j in range(40):
        pages.K[pages.table[0, j]] = level[j]
    q = torch.ones((1, 2, 64))
    bounds = torch.zeros((pages.K.shape[0], 1, 2, 64))
    got, b = run(pages, q, bounds, lens, 20, gpu_device, since=[0])
    assert got.flatten().tolist() == sorted([j for j in range(40) if j % 4 == 3] + [j for j in range(40) if j % 4 in (1, 2)][:10])
    for j in range(40):
        pages.K[pages.table[0, j]] = -0.0 if j % 2 else 0.0
    got, _ = run(pages, q, bounds, lens, 7, gpu_device, since=[0])
    assert got.flatten().tolist() == [0, 1, 2, 3, 4, 5, 39]


def test_values_that_are_not_finite(gpu_device):
    """A NaN row puts its page first and its bounds stay NaN; infinities score as such; a query that is NaN leaves the lowest pages."""
    lens = [30 * 16, 30 * 16]
    pages = Pages(lens, 4, 2, 64, 16, "bf16", gpu_device)
    pages.K[pages.table[0, 11], 0, 3, 5] = float("nan")
    pages.K[pages.table[0, 20], 1, 3, 5] = float("inf")
    pages.K[pages.table[0, 21], 1, 3, 5] = -float("inf")
    pages.q[0, 2:, 5] = 1.0
    pages.q[1, 0, 7] = float("nan")
    bounds = torch.zeros((pages.K.shape[0], 2, 2, 64), dtype=torch.bfloat16)
    got, b = run(pages, pages.q, bounds, lens, 4, gpu_device, since=[0, 0])
    want = reference_bounds(pages, lens, [0, 0], bounds)
    assert same(b, want) and torch.equal(got, reference_lists(pages, pages.q, want, lens, 4, 0, 1))
    assert 11 in got[0, 0] and {20, 21} <= set(got[0, 1].tolist()) and got[1, 0].tolist() == [0, 1, 2, 29]
    # a later row of the page does not wash it out
    more, b2 = run(pages, pages.q, b, [12 * 16, 5], 4, gpu_device, since=[12 * 16 - 2, 4])
    assert b2[pages.table[0, 11], 0, :, 5].isnan().all() and 11 in more[0, 0]


def test_pages_outside_the_pool_and_full_tables(gpu_device):
    lens = [25 * 16, 1000]
    pages = Pages([25 * 16, 25 * 16], 4, 2, 64, 16, "f16", gpu_device, table_pages=25)
    for j, page in ((2, -1), (3, 1 << 30), (24, -7), (9, pages.K.shape[0])):
        pages.table[0, j] = page
    bounds = torch.zeros((pages.K.shape[0], 2, 2, 64), dtype=torch.float16)
    got, b = run(pages, pages.q, bounds, lens, 6, gpu_device, since=[0, 0])
    want = reference_bounds(pages, lens, [0, 0], bounds)
    assert same(b, want)
    lists = reference_lists(pages, pages.q, want, lens, 6, 0, 1)
    assert torch.equal(got, lists) and 24 in lists[0, 0] and not {2, 3, 9} & set(lists[0].flatten().tolist())
    # more pages wanted than have a score: the lowest of the others
    got, _ = run(pages, pages.q, want, lens, 23, gpu_device)
    assert torch.equal(got, reference_lists(pages, pages.q, want, lens, 23, 0, 1)) and 2 in got[0, 0] and 3 not in got[0, 0]
    # positions past the table: the newest token has no row, its page is none
    again, b2 = run(pages, pages.q, want, [400, 1000], 6, gpu_device)
    assert same(b2, want)


@pytest.mark.parametrize("table_pages,budget", [(700, 300), (5000, 16), (20000, 19990)])
def test_long_tables(table_pages, budget, gpu_device):
    """Many workgroups a pair, keys close together, almost all or almost none chosen; the pool is shared, so that only the table is long."""
    rng = np.random.default_rng(budget)
    K = torch.zeros((900, 1, 16, 64))
    bounds = torch.from_numpy(rng.standard_normal((900, 1, 1, 64)).astype(np.float32)).abs().mul(torch.tensor([-1.0, 1.0]).view(1, 1, 2, 1))
    bounds[100:200] = bounds[100]
    table = torch.from_numpy(rng.integers(0, 900, (2, table_pages)).astype(np.int32))
    ctx = torch.tensor([table_pages * 16, table_pages * 16 - 35], dtype=torch.int32)
    q = torch.from_numpy(rng.standard_normal((2, 4, 64)).astype(np.float32))
    got = span.paged_select(q.to(gpu_device), K.to(gpu_device), bounds.to(gpu_device), table.to(gpu_device), ctx.to(gpu_device), budget,
                            since=ctx.to(gpu_device)).cpu()
    for b in range(2):
        want = select(q[b].double().numpy(), bounds[:, 0].double().numpy(), int(ctx[b]), table[b].tolist(), 16, budget, 0, 1)
        assert got[b, 0].tolist() == want


def test_bounds_and_lists_beyond_four_gib(gpu_device):
    """Pools whose rows, and bounds whose entries, lie past 32 bits."""
    N, KV, P, D = 70000, 64, 16, 128
    K = torch.empty((N, KV, P, D), device=gpu_device)
    V = K
    bounds = torch.empty((N, KV, 2, D), device=gpu_device)
    assert bounds.numel() * 4 > 1 << 32
    g = torch.Generator(device=gpu_device).manual_seed(0)
    table = torch.tensor([[N - 1, 3, N - 2, N // 2, 5, N // 3]], dtype=torch.int32, device=gpu_device)
    for page in table.flatten().tolist():
        K[page] = torch.randn((KV, P, D), generator=g, device=gpu_device)
    q = torch.randn((1, KV, D), generator=g, device=gpu_device)
    ctx = torch.tensor([90], dtype=torch.int32, device=gpu_device)
    got = span.paged_select(q, K, bounds, table, ctx, 3, since=torch.zeros(1, dtype=torch.int32, device=gpu_device))
    where = table[0].long()
    rows = K[where]
    rows[5, :, 10:] = rows[5, :, :1]
    assert torch.equal(bounds[where, :, 0], rows.amin(2)) and torch.equal(bounds[where, :, 1], rows.amax(2))
    small = bounds[where].cpu().double().numpy()
    for h in range(KV):
        assert got[0, h].tolist() == select(q[0, h:h + 1].cpu().double().numpy(), small[:, h], 90, range(6), 16, 3, 0, 1)
    out = span.paged_selected_decode_attn(q, K, V, table, ctx, got, 0.1).cpu().double()
    for h in range(KV):
        p = [p for j in got[0, h].tolist() for p in range(j * 16, min(j * 16 + 16, 90))]
        k, v = (x[where][:, h].reshape(-1, D)[p].cpu().double() for x in (K, V))
        w = torch.softmax(k @ q[0, h].cpu().double() * 0.1, 0)
        assert float((out[0, h] - w @ v).abs().max()) < 1e-4


@pytest.mark.parametrize("dtype,bound", [("f32", 1e-5), ("f16", 2e-5), ("bf16", 2e-5)])
@pytest.mark.parametrize("heads,kv_heads,head_dim,page", [(4, 4, 64, 16), (16, 1, 128, 16), (14, 2, 64, 64), (6, 3, 128, 256)])
@pytest.mark.parametrize("splits", [0, 5])
def test_selected_attention(dtype, bound, heads, kv_heads, head_dim, page, splits, gpu_device):
    """Lists as the selection makes them, in other orders, with entries that are none; each KV head its own.  (The bounds are those of one-token attention in general:
    scores of some tens, exact 16-bit products, fp32 sums.)"""
    lens = [0, 1, 3 * page + 5, 8 * page, 20 * page + 1, 40 * page - 3]
    pages = Pages(lens, heads, kv_heads, head_dim, page, dtype, gpu_device, seed=page)
    K, V, table, ctx = pages.to("K", "V", "table", "ctx")
    rng = np.random.default_rng(1)
    budget = 9
    lists = np.full((len(lens), kv_heads, budget), -1, np.int32)
    for b, n in enumerate(lens):
        for h in range(kv_heads):
            count = -(-n // page)
            some = rng.permutation(count)[:budget]
            if h % 2 == 0:
                some = np.sort(some)
            lists[b, h, :len(some)] = some
            if count > budget and h == 0:
                lists[b, h, 3], lists[b, h, 5] = -1, count + 100000  # entries that are none of the sequence's
    out = span.paged_selected_decode_attn(pages.q.to(gpu_device), K, V, table, ctx, torch.from_numpy(lists).to(gpu_device), head_dim ** -0.5, num_splits=splits)
    G = heads // kv_heads
    for b, n in enumerate(lens):
        for h in range(kv_heads):
            p = [p for j in lists[b, h] if 0 <= j < -(-n // page) for p in range(j * page, min((j + 1) * page, n))]
            want, _ = attend(pages, pages.K, pages.V, b, pages.q[b], p, head_dim ** -0.5)
            assert float((out[b, h * G:(h + 1) * G].cpu().double() - want[h * G:(h + 1) * G]).abs().max()) <= bound, (b, h)


def test_all_pages_selected_is_the_whole_cache(gpu_device):
    pages = Pages([500, 33, 1], 8, 2, 128, 16, "bf16", gpu_device)
    K, V, table, ctx = pages.to("K", "V", "table", "ctx")
    every = torch.arange(40, dtype=torch.int32, device=gpu_device).expand(3, 2, 40).contiguous()
    got = span.paged_selected_decode_attn(pages.q.to(gpu_device), K, V, table, ctx, every, 0.1, num_splits=2)
    whole = span.paged_decode_attn(pages.q.to(gpu_device), K, V, table, ctx, 0.1, num_splits=2)
    assert float((got - whole).abs().max()) <= 2e-5
