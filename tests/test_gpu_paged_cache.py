"""Rows into and out of a cache in pages: append and evict move bits and count, so everything has to be equal."""
import numpy as np
import pytest
import torch

import paper_2404_09336_amd as span
from paged_reference import DTYPES, Pages, evict

pytestmark = pytest.mark.gpu


def same(a, b):
    """The same bits, NaN among them."""
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("kv_heads,head_dim", [(1, 64), (3, 128), (32, 128)])
@pytest.mark.parametrize("new", ["one", "some"])
@pytest.mark.parametrize("track", [False, True])
def test_append(dtype, kv_heads, head_dim, new, track, gpu_device):
    """One token each, or 0 to 70 across pages; more new tokens than positions drop the first; rows that are nobody's; pages outside the pool."""
    lens = [5, 16, 17, 100, 64, 1, 90, 3]
    t = [1] * 8 if new == "one" else [5, 0, 1, 70, 33, 1, 20, 7]  # (the last has 7 new tokens at 3 positions)
    pages = Pages(lens, kv_heads, kv_heads, head_dim, 16, dtype, gpu_device, seed=kv_heads)
    pages.table[6, 5] = -1
    pages.table[4, 3] = pages.K.shape[0]
    spare = 0 if new == "one" else 4
    total = sum(t) + spare                            # the last rows are nobody's
    k_new, v_new = (torch.randn((total, kv_heads, head_dim), generator=pages.generator).to(DTYPES[dtype]) for _ in range(2))
    off = np.cumsum([0] + t).astype(np.int32)
    positions = torch.full((8, kv_heads, pages.capacity), -9, dtype=torch.int32)
    seen = torch.tensor(lens, dtype=torch.int32) + 1000 * torch.arange(8, dtype=torch.int32)
    K, V, table, ctx = pages.to("K", "V", "table", "ctx")
    pos = positions.to(gpu_device)
    kw = {"positions": pos, "seen": seen.to(gpu_device)} if track else {}
    span.paged_append(k_new.to(gpu_device), v_new.to(gpu_device), K, V, table, ctx,
                      None if new == "one" else torch.from_numpy(off).to(gpu_device), **kw)
    for b in range(8):
        for j in range(t[b]):
            p, row = lens[b] - t[b] + j, int(off[b]) + j
            if p < 0:
                continue
            positions[b, :, p] = p + 1000 * b
            page = int(pages.table[b, p // 16])
            if 0 <= page < pages.K.shape[0]:
                pages.K[page, :, p % 16], pages.V[page, :, p % 16] = k_new[row], v_new[row]
    assert same(K.cpu(), pages.K) and same(V.cpu(), pages.V)
    if track:
        assert torch.equal(pos.cpu(), positions)


@pytest.mark.parametrize("batch", [64, 65, 300, 4097])
def test_append_finds_the_sequence(batch, gpu_device):
    """Batches beyond a wave's 64 and 64 * 64 sequences, many of them without a new token."""
    rng = np.random.default_rng(batch)
    t = rng.integers(0, 3, batch) * (rng.random(batch) < 0.5)
    t[0], t[-1] = 2, 1
    off = np.cumsum(np.concatenate([[0], t])).astype(np.int32)
    D, P = 64, 16
    K, V = (torch.zeros((batch, 1, P, D), dtype=torch.float16, device=gpu_device) for _ in range(2))
    table = torch.arange(batch, dtype=torch.int32, device=gpu_device).flip(0)[:, None].contiguous()
    ctx = torch.full((batch,), 9, dtype=torch.int32, device=gpu_device)
    k_new = torch.arange(1, int(off[-1]) + 1, device=gpu_device).half()[:, None, None].expand(-1, 1, D).contiguous()
    span.paged_append(k_new, -k_new, K, V, table, ctx, torch.from_numpy(off).to(gpu_device))
    want = torch.zeros((batch, P), dtype=torch.float16)  # (as the rows are: from 2048 on fp16 holds even numbers only)
    for b in range(batch):
        for j in range(t[b]):
            want[batch - 1 - b, 9 - t[b] + j] = off[b] + j + 1
    assert torch.equal(K[:, 0, :, 5].cpu(), want) and torch.equal(V[:, 0, :, 63].cpu(), -want)


def run_evict(pages, weights, positions, budget, sinks, recent, in_place, gpu_device):
    """Runs the call and compares everything with the plain form."""
    B, KV, cap, P = len(pages.lens), pages.kv_heads, pages.capacity, pages.page
    K, V, table, ctx = pages.to("K", "V", "table", "ctx")
    w = weights.to(gpu_device)
    pos = None if positions is None else positions.to(gpu_device)
    if in_place:
        got = span.paged_evict(K, V, table, ctx, w, budget, sinks=sinks, recent=recent, positions=pos, weights_out=w, positions_out=pos, new_lens=ctx)
    else:
        got = span.paged_evict(K, V, table, ctx, w, budget, sinks=sinks, recent=recent, positions=pos)
        assert same(w.cpu(), weights) and (pos is None or torch.equal(pos.cpu(), positions)) and torch.equal(ctx.cpu(), pages.ctx)
    want_w = weights.clone() if in_place else torch.zeros_like(weights)
    want_p = None if positions is None else (positions.clone() if in_place else torch.full_like(positions, -1))
    moved = 0
    for b in range(B):
        n = pages.lens[b]
        for h in range(KV):
            wn = weights[b, h, :n].numpy()
            pn = np.arange(n) if positions is None else positions[b, h, :n].numpy()
            to, of = evict(n, wn, pn, budget, sinks, recent)
            moved += len(to)
            left = min(n, budget)
            for out, src, none in ((want_w, weights, 0.0), (want_p, positions, -1)):
                if out is None:
                    continue
                out[b, h, :left] = src[b, h, :left]
                out[b, h, left:n] = none
                out[b, h, to] = src[b, h, of]
            for d, s in zip(to, of):
                for pool in (pages.K, pages.V):
                    pool[pages.table[b, d // P], h, d % P] = pool[pages.table[b, s // P], h, s % P]
    assert same(K.cpu(), pages.K) and same(V.cpu(), pages.V)
    assert same(got[0].cpu(), want_w)
    assert got[1] is None if positions is None else torch.equal(got[1].cpu(), want_p)
    assert got[2].tolist() == [min(n, budget) for n in pages.lens]
    return moved


@pytest.mark.parametrize("dtype,head_dim", [("f32", 128), ("f32", 64), ("f16", 64), ("bf16", 128)])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("with_positions", [False, True])
def test_evict(dtype, head_dim, in_place, with_positions, gpu_device):
    """Sequences below, at and above the budget; few distinct weights, so that ties are broken by the slot; positions in any order."""
    pages = Pages([0, 1, 99, 100, 101, 163, 400, 1000], 3, 3, head_dim, 32, dtype, gpu_device, seed=1)
    g = torch.Generator().manual_seed(2)
    weights = torch.randint(0, 6, (8, 3, pages.capacity), generator=g).float() / 4
    positions = torch.rand((8, 3, pages.capacity), generator=g).argsort(dim=-1).to(torch.int32) if with_positions else None
    assert run_evict(pages, weights, positions, 100, 3, 20, in_place, gpu_device) > 100


@pytest.mark.parametrize("sinks,recent,budget", [(0, 0, 1), (1, 0, 1), (0, 1, 1), (0, 64, 64), (4, 60, 64), (0, 0, 299), (7, 0, 1000)])
def test_evict_budgets(sinks, recent, budget, gpu_device):
    """A budget of one row, all of it protected, one row less than there is, more than there is."""
    pages = Pages([300, 64, 65], 2, 2, 64, 16, "f16", gpu_device, seed=4)
    g = torch.Generator().manual_seed(budget)
    weights = torch.rand((3, 2, pages.capacity), generator=g)
    run_evict(pages, weights, None, budget, sinks, recent, False, gpu_device)


def test_evict_orders_every_float(gpu_device):
    """Negative and infinite weights, denormals, both zeros (equal), NaN of either sign below all others."""
    pages = Pages([512], 1, 1, 64, 16, "f16", gpu_device, seed=6)
    kinds = torch.tensor([float("nan"), -float("nan"), float("-inf"), -3e38, -1.0, -1e-42, -0.0, 0.0, 1e-45, 1e-38, 1.0, 1.0000001, 3e38, float("inf")])
    g = torch.Generator().manual_seed(0)
    weights = kinds[torch.randint(0, len(kinds), (1, 1, 512), generator=g)]
    weights[0, 0, :4] = torch.tensor([-2147483648, 2147483647, -1, 0x7f800001], dtype=torch.int64).to(torch.int32).view(torch.float32)
    for budget in (40, 110, 200, 250, 300, 400, 480):
        run_evict(Pages([512], 1, 1, 64, 16, "f16", gpu_device, seed=6), weights, None, budget, 0, 0, False, gpu_device)
    assert pages.capacity == 512


@pytest.mark.parametrize("n,cap_pages", [(8192, 512), (8200, 513), (32768, 2048), (40000, 2500)])
def test_evict_long(n, cap_pages, gpu_device):
    """On both sides of what the keys in LDS hold."""
    pages = Pages([n, 2000], 1, 1, 64, 16, "f16", gpu_device, seed=3, table_pages=cap_pages)
    g = torch.Generator().manual_seed(n)
    weights = torch.rand((2, 1, pages.capacity), generator=g).pow(8)
    positions = torch.rand((2, 1, pages.capacity), generator=g).argsort(dim=-1).to(torch.int32)
    for in_place in (False, True):
        run_evict(pages, weights, positions, 1500, 4, 700, in_place, gpu_device)
        pages = Pages([n, 2000], 1, 1, 64, 16, "f16", gpu_device, seed=3, table_pages=cap_pages)


@pytest.mark.parametrize("batch,kv_heads", [(1, 1), (3, 5), (20, 16)])
@pytest.mark.parametrize("cap_pages", [100, 400, 700, 1100])
def test_evict_again_and_again_in_place(batch, kv_heads, cap_pages, gpu_device):
    """One call after the other on one workspace, on the arrays themselves, with fewer and more (sequence, KV head) pairs than a card has CUs; the last
    pages of the tables are free.  A sequence below the budget, one of one row, one without any."""
    lens = ([1500, 900, 1, 0, 1201] * 4)[:batch]
    pages = Pages(lens, kv_heads, kv_heads, 64, 16, "f16", gpu_device, seed=batch, table_pages=94)
    table = torch.cat((pages.table, torch.full((batch, cap_pages - 94), -1, dtype=torch.int32)), dim=1).to(gpu_device)
    cap, budget = cap_pages * 16, 1000
    g = torch.Generator().manual_seed(cap)
    weights = torch.rand((batch, kv_heads, cap), generator=g)
    positions = torch.rand((batch, kv_heads, cap), generator=g).argsort(dim=-1).to(torch.int32)
    K, V, ctx = pages.to("K", "V", "ctx")
    w, pos = weights.to(gpu_device), positions.to(gpu_device)
    call = span.prepare_paged_evict(K, V, table, ctx, w, budget, sinks=2, recent=30, positions=pos, weights_out=w, positions_out=pos, new_lens=ctx)
    want = None
    for _ in range(4):
        for x, y in ((K, pages.K), (V, pages.V), (ctx, pages.ctx), (w, weights), (pos, positions)):
            x.copy_(y)
        call()
        torch.cuda.synchronize()
        got = [x.cpu() for x in (K, V, ctx, w, pos)]
        assert got[2].tolist() == [min(n, budget) for n in lens]
        if want is None:
            want = got
            for b in range(0, batch, 4):
                for h in (0, kv_heads - 1):
                    n = lens[b]
                    to, of = evict(n, weights[b, h, :n].numpy(), positions[b, h, :n].numpy(), budget, 2, 30)
                    expect = weights[b, h].clone()
                    expect[to] = weights[b, h][of]
                    expect[min(n, budget):n] = 0.0
                    assert same(got[3][b, h], expect)
                    for d, s in zip(to, of):
                        assert same(got[0][pages.table[b, d // 16], h, d % 16], pages.K[pages.table[b, s // 16], h, s % 16])
        for x, y in zip(got, want):
            assert same(x, y)


def test_a_life_of_a_cache(gpu_device):
    """Together, as a program uses them, step by step in one captured graph per step: rows go in, a token attends and the weights add up; an eviction
    whenever a cache outgrows its budget.  The plain form follows on the host."""
    from paged_reference import attend
    B, H, KV, D, P, budget, recent, sinks = 2, 4, 2, 64, 16, 40, 8, 2
    pages = Pages([30, 12], H, KV, D, P, "f32", gpu_device, seed=12, table_pages=4)
    K, V, table, ctx = pages.to("K", "V", "table", "ctx")
    cap = pages.capacity
    weights = torch.zeros((B, KV, cap), device=gpu_device)
    positions = torch.arange(cap, dtype=torch.int32, device=gpu_device).expand(B, KV, cap).contiguous()
    seen = ctx.clone()
    k_new, v_new, q = (torch.zeros((B, n, D), device=gpu_device) for n in (KV, KV, H))
    side = torch.cuda.Stream(device=gpu_device)
    append = span.prepare_paged_append(k_new, v_new, K, V, table, ctx, positions=positions, seen=seen, stream=side.cuda_stream)
    attend_call = span.prepare_paged_decode_attn(q, K, V, table, ctx, D ** -0.5, weights=weights, stream=side.cuda_stream)
    cut = span.prepare_paged_evict(K, V, table, ctx, weights, budget, sinks=sinks, recent=recent, positions=positions, weights_out=weights,
                                   positions_out=positions, new_lens=ctx, stream=side.cuda_stream)
    torch.cuda.synchronize()
    step, shrink = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(step, stream=side):
        ctx.add_(1)
        seen.add_(1)
        append()
        attend_call()
    with torch.cuda.graph(shrink, stream=side):
        cut()
    w_host = np.zeros((B, KV, cap))
    for t in range(60):
        new = [torch.randn(x.shape, generator=pages.generator) for x in (k_new, v_new, q)]
        for x, y in zip((k_new, v_new, q), new):
            x.copy_(y)
        torch.cuda.synchronize()
        step.replay()
        torch.cuda.synchronize()
        now = ctx.tolist()
        K_host, V_host = K.cpu(), V.cpu()
        for b in range(B):
            p = now[b] - 1
            assert torch.equal(K_host[pages.table[b, p // P], :, p % P], new[0][b]) and torch.equal(V_host[pages.table[b, p // P], :, p % P], new[1][b])
            assert positions[b, :, p].tolist() == [seen[b].item() - 1] * KV
            out, w = attend(pages, K_host, V_host, b, new[2][b], range(now[b]), D ** -0.5)
            assert float((attend_call.out[b].cpu().double() - out).abs().max()) <= 1e-5
            w_host[b, :, :now[b]] += w.numpy()
        # up to 60 additions, each off by its weights' error (1e-5 of at most 2) and half a step of a sum of at most 120
        assert np.abs(weights.cpu().numpy() - w_host).max() <= 60 * (2e-5 + 120 * 2.0 ** -24)
        if max(now) == cap:
            w_dev, p_dev = weights.cpu(), positions.cpu()
            lists = {}
            for b in range(B):
                for h in range(KV):
                    lists[b, h] = evict(now[b], w_dev[b, h, :now[b]].numpy(), p_dev[b, h, :now[b]].numpy(), budget, sinks, recent)
            shrink.replay()
            torch.cuda.synchronize()
            for (b, h), (to, of) in lists.items():
                w_host[b, h, to] = w_host[b, h, of]
                w_host[b, h, min(now[b], budget):] = 0
                kept = positions[b, h, :min(now[b], budget)].tolist()
                total = seen[b].item()
                if now[b] > budget:
                    assert set(range(sinks)) <= set(kept) and set(range(total - recent, total)) <= set(kept)
                for d, s in zip(to, of):
                    assert torch.equal(K[pages.table[b, d // P], h, d % P].cpu(), K_host[pages.table[b, s // P], h, s % P])
            assert ctx.tolist() == [min(n, budget) for n in now]
    assert min(seen.tolist()) == 72
