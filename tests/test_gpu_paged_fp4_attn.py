"""One-token attention over pages of 4-bit values against the same in 64 bits over the values that the pages hold."""
import numpy as np
import pytest
import torch

import paper_2404_09336_amd as span
from paged_more_reference import from_fp4, place, pool_fp4, read_fp4
from paged_reference import DTYPES, seen_positions

pytestmark = pytest.mark.gpu


class Fp4Pages:
    """Random pools in random page order; what no sequence holds, and the rows past a sequence's length, are NaN."""

    def __init__(self, lens, heads, kv_heads, head_dim, page, dtype, device, seed=0, table_pages=None, spread=0):
        self.lens, self.heads, self.kv_heads, self.head_dim, self.page = list(lens), heads, kv_heads, head_dim, page
        rng = np.random.default_rng(seed)
        B = len(self.lens)
        self.table_pages = table_pages or max(1, max(-(-n // page) for n in self.lens))
        N = B * self.table_pages + 3
        self.table = torch.from_numpy(rng.permutation(N)[:B * self.table_pages].reshape(B, self.table_pages).astype(np.int32))
        self.pools, self.values = [], []
        for is_v in (False, True):
            x = np.full((N, kv_heads, page, head_dim), np.nan)
            for b, n in enumerate(self.lens):
                for i in range(-(-min(n, self.capacity) // page)):
                    rows = min(page, n - i * page)
                    scale = 2.0 ** rng.integers(-spread, spread + 1, (kv_heads, rows, head_dim // 32)).repeat(32, -1)
                    x[self.table[b, i], :, :rows] = rng.standard_normal((kv_heads, rows, head_dim)) * scale
            self.pools.append(torch.from_numpy(pool_fp4(x, is_v)).to(device))
            self.values.append(read_fp4(self.pools[-1].cpu().numpy(), is_v))
        self.q = torch.from_numpy(rng.standard_normal((B, heads, head_dim))).to(DTYPES[dtype])
        self.device, self.ctx = device, torch.tensor(self.lens, dtype=torch.int32)

    @property
    def capacity(self):
        return self.table_pages * self.page

    def cache(self):
        return (*self.pools, self.table.to(self.device))

    def attend(self, b, positions, scale, q=None):
        """(out [heads, head_dim], tolerance of each value) in 64 bits."""
        H, KV, D = self.heads, self.kv_heads, self.head_dim
        if len(positions) == 0:
            return np.zeros((H, D)), np.zeros((H, D))
        p = np.asarray(positions, np.int64)
        page = self.table[b].numpy()[p // self.page]
        k, v = (x[page, :, p % self.page].transpose(1, 0, 2) for x in self.values)  # [KV, n, D]
        q = (self.q[b] if q is None else q).double().numpy().reshape(KV, H // KV, D)
        s = scale * q @ k.transpose(0, 2, 1)
        w = np.exp(s - s.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        # A channel of q is off by half a unit of its last digit at most: 2^-21 of the power of two above its block's largest (2^-20 of the largest); the sums of a score
        # round to fp32 a few times, and so does its product with the scale.  A weight is off relatively by twice the largest difference of scores.
        block = np.abs(q).reshape(KV, H // KV, -1, 32).max(-1, keepdims=True) * np.ones(32)
        digit = np.abs(scale) * (block.reshape(q.shape) @ np.abs(k).transpose(0, 2, 1)) * 2.0 ** -20
        sums = np.abs(scale) * (np.abs(q) @ np.abs(k).transpose(0, 2, 1)) * 2.0 ** -20
        off = np.expm1(2 * (digit + sums).max(-1, keepdims=True))
        # A weight goes in as two bf16 terms, each rounded by half a step (2^-9) at most: 2^-18 of it is lost.  Products with V are exact, their sums round: up to three a step of 32
        # positions of a wave, the joins of waves and slices.
        chain = 2.0 ** -18 + (3 * (len(p) // 32 + 1) + 64) * 2.0 ** -24
        return (w @ v).reshape(H, D), ((off + chain) * (w @ np.abs(v))).reshape(H, D) + 1e-30


def check(pages, out, b, positions, scale, q=None):
    want, bound = pages.attend(b, positions, scale, q)
    got = out[b].cpu().double().numpy()
    assert np.all(np.abs(got - want) <= bound), (b, len(positions), float(np.abs(got - want).max()), float(bound.min()))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads,kv_heads,head_dim", [(4, 4, 64), (16, 1, 128), (14, 2, 64), (5, 5, 128), (12, 4, 128)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (40, 4), (15, 17), (100, 64)])
def test_lengths_and_windows(dtype, heads, kv_heads, head_dim, window, sinks, gpu_device):
    """No position to a few hundred, around the edges of units, steps and slices; windows and sinks that meet in a unit."""
    lens = [0, 1, 15, 16, 17, 31, 32, 33, 63, 65, 127, 129, 255, 257, 400]
    pages = Fp4Pages(lens, heads, kv_heads, head_dim, 16, dtype, gpu_device, seed=heads, spread=3)
    out = span.paged_decode_attn_fp4(pages.q.to(gpu_device), *pages.cache(), pages.ctx.to(gpu_device), head_dim ** -0.5, window=window, sinks=sinks)
    for b, n in enumerate(lens):
        check(pages, out, b, seen_positions(n, window, sinks), head_dim ** -0.5)


@pytest.mark.parametrize("page", [16, 64, 1024])
@pytest.mark.parametrize("splits", [0, 1, 3, 40])
@pytest.mark.parametrize("head_dim", [64, 128])
def test_slices(page, splits, head_dim, gpu_device):
    """Long, short and empty sequences, by the library's slices and by given ones; more than 64 units of a wave."""
    lens = [9000, 0, 130, 4111, 1, 700]
    pages = Fp4Pages(lens, 8, 2, head_dim, page, "bf16", gpu_device, seed=page)
    out = span.paged_decode_attn_fp4(pages.q.to(gpu_device), *pages.cache(), pages.ctx.to(gpu_device), 0.2, num_splits=splits)
    for b, n in enumerate(lens):
        check(pages, out, b, range(n), 0.2)


@pytest.mark.parametrize("batch", [65, 130, 600])
def test_many_sequences(batch, gpu_device):
    """More than a wave's lanes, and more than those whose slices are looked for."""
    rng = np.random.default_rng(batch)
    lens = rng.integers(0, 300, batch).tolist()
    pages = Fp4Pages(lens, 2, 1, 64, 16, "f16", gpu_device, seed=batch)
    out = span.paged_decode_attn_fp4(pages.q.to(gpu_device), *pages.cache(), pages.ctx.to(gpu_device), 0.125)
    for b, n in enumerate(lens):
        check(pages, out, b, range(n), 0.125)


SPANS = {"some": [[(0, 20), (33, 34), (50, 51), (60, 200)], [], [(5, 6)], [(0, 16), (16, 32), (32, 33)], [(3, 13), (13, 17), (17, 18), (18, 299)], [(299, 300)]],
         "edges": [[(15, 17)], [(16, 32)], [(0, 1), (2, 3), (4, 5), (6, 7), (8, 9), (10, 11), (12, 13), (14, 15)], [(31, 33), (47, 49)], [(0, 300)], [(7, 7), (8, 8), (9, 10)]],
         "many": [[(4 * i, 4 * i + 1 + i % 3) for i in range(75)], [(2 * i, 2 * i + 1) for i in range(150)], [(4 * i, 4 * i + 3) for i in range(64)], [(0, 300)], [], [(1, 2)]]}


@pytest.mark.parametrize("which", list(SPANS))
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads,kv_heads,head_dim", [(4, 4, 128), (16, 2, 64)])
@pytest.mark.parametrize("told", [False, True])
def test_spans(which, dtype, heads, kv_heads, head_dim, told, gpu_device):
    """Intervals that share units, empty ones, more than 64; with the counts of the host and without."""
    lists = SPANS[which]
    pages = Fp4Pages([300] * len(lists), heads, kv_heads, head_dim, 32, dtype, gpu_device, seed=7)
    off = np.cumsum([0] + [len(x) for x in lists]).astype(np.int32)
    st, en = (np.asarray([iv[i] for x in lists for iv in x], np.int32) for i in (0, 1))
    tokens = np.asarray([sum(e - s for s, e in x) for x in lists], np.int64)
    args = [torch.from_numpy(x).to(gpu_device) for x in (off, st, en)]
    out = span.paged_span_decode_attn_fp4(pages.q.to(gpu_device), *pages.cache(), *args, 0.1, tokens_per_seq=tokens if told else None)
    for b, x in enumerate(lists):
        check(pages, out, b, [p for s, e in x for p in range(s, e)], 0.1)


def test_long_span_lists(gpu_device):
    """Thousands of intervals: many chunks of them, slices from a table, windows of units beyond a wave's first."""
    rng = np.random.default_rng(3)
    lists = []
    for n in (12000, 40, 7000):
        cuts = np.sort(rng.choice(n, min(n // 4 * 2, 5000), replace=False))
        lists.append([(int(a), int(b)) for a, b in zip(cuts[::2], cuts[1::2])])
    pages = Fp4Pages([12000, 40, 7000], 4, 2, 64, 64, "bf16", gpu_device, seed=9)
    off = np.cumsum([0] + [len(x) for x in lists]).astype(np.int32)
    st, en = (np.asarray([iv[i] for x in lists for iv in x], np.int32) for i in (0, 1))
    tokens = np.asarray([sum(e - s for s, e in x) for x in lists], np.int64)
    args = [torch.from_numpy(x).to(gpu_device) for x in (off, st, en)]
    for kw in ({}, {"tokens_per_seq": tokens}, {"num_splits": 1}):
        out = span.paged_span_decode_attn_fp4(pages.q.to(gpu_device), *pages.cache(), *args, 0.3, **kw)
        for b, x in enumerate(lists):
            check(pages, out, b, [p for s, e in x for p in range(s, e)], 0.3)


def test_lists_that_are_not_valid_touch_nothing_else(gpu_device):
    """Ends ahead of starts, positions past the table, overlaps, offsets that go back: whatever comes out, valid sequences beside them are right."""
    lists = [[(250, 100), (-5, 20), (290, 5000)], [(0, 300), (0, 300), (0, 300)], [(10, 60)], [(1 << 30, (1 << 31) - 1)]]
    pages = Fp4Pages([300] * 4, 4, 2, 64, 16, "f16", gpu_device)
    off = np.cumsum([0] + [len(x) for x in lists]).astype(np.int32)
    st, en = (np.asarray([iv[i] for x in lists for iv in x], np.int32) for i in (0, 1))
    args = [torch.from_numpy(x).to(gpu_device) for x in (off, st, en)]
    out = span.paged_span_decode_attn_fp4(pages.q.to(gpu_device), *pages.cache(), *args, 0.3)
    check(pages, out, 2, range(10, 60), 0.3)
    back = torch.tensor([3, 0, 9999, -4, 2], dtype=torch.int32, device=gpu_device)
    span.paged_span_decode_attn_fp4(pages.q.to(gpu_device), *pages.cache(), back, *args[1:], 0.3)
    torch.cuda.synchronize()


@pytest.mark.parametrize("head_dim", [64, 128])
def test_pages_outside_the_pool_and_full_tables(head_dim, gpu_device):
    lens = [200, 90, 300]  # the last has more positions than its table: nobody attends those
    pages = Fp4Pages(lens, 4, 2, head_dim, 16, "f32", gpu_device, table_pages=13)
    pages.table[0, 2], pages.table[0, 12], pages.table[1, 0] = -1, pages.pools[0].shape[0], 1 << 30
    out = span.paged_decode_attn_fp4(pages.q.to(gpu_device), *pages.cache(), pages.ctx.to(gpu_device), 0.125)
    there = [[p for p in range(200) if p // 16 not in (2, 12)], list(range(16, 90)), list(range(208))]
    for b in range(3):
        check(pages, out, b, there[b], 0.125)
    windowed = span.paged_decode_attn_fp4(pages.q.to(gpu_device), *pages.cache(), pages.ctx.to(gpu_device), 0.125, window=100, sinks=20)
    check(pages, windowed, 2, list(range(20)) + list(range(200, 208)), 0.125)  # (a window goes by the token's own position, 299)
    out = span.paged_decode_attn_fp4(pages.q.to(gpu_device), *pages.cache(), torch.tensor([-3, 0, 1], dtype=torch.int32, device=gpu_device), 0.125)
    assert not out[:2].any() and out[2].any()


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("where", ["k", "v"])
def test_a_block_that_is_nan(where, head_dim, gpu_device):
    """Reaches the rows that attend it and nobody else: the other KV head, other sequences, the same position outside the window."""
    pages = Fp4Pages([100, 100], 8, 2, head_dim, 16, "bf16", gpu_device)
    pool = pages.pools[where == "v"]
    codes, exps = place(16, head_dim, 37 % 16, where == "v")
    flat = pool.view(pool.shape[0], 2, -1)
    flat[int(pages.table[0, 2]), 1, int(exps[1])] = 255
    args = (pages.q.to(gpu_device), *pages.cache(), pages.ctx.to(gpu_device), 0.125)
    out = span.paged_decode_attn_fp4(*args)
    assert not out[0, :4].isnan().any() and not out[1].isnan().any()
    assert out[0, 4:].isnan().all() if where == "k" else out[0, 4:, 32:64].isnan().all() and not out[0, 4:, :32].isnan().any()
    assert not span.paged_decode_attn_fp4(*args, window=62, sinks=37).isnan().any()
    assert span.paged_decode_attn_fp4(*args, window=63).isnan().any() and span.paged_decode_attn_fp4(*args, window=5, sinks=38).isnan().any()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("scale", [0.125, -0.5, 0.0, 3.7, 1e-30])
def test_scales_and_sizes_of_queries(dtype, scale, gpu_device):
    """Query rows of very different size within a row and a group, zeros, the type's least numbers; scales of either sign."""
    pages = Fp4Pages([333, 20], 16, 2, 64, 16, dtype, gpu_device, spread=5)
    q = pages.q.double()
    q[0, 0] = 0
    q[0, 1, ::2] *= 2.0 ** -12
    q[0, 2, :32] *= 2.0 ** -9
    q[0, 3] *= 2.0 ** -24 if dtype == "f16" else 2.0 ** -120
    q[0, 4, 0], q[0, 5, 40] = 100.0, -200.0
    pages.q = q.to(DTYPES[dtype])
    out = span.paged_decode_attn_fp4(pages.q.to(gpu_device), *pages.cache(), pages.ctx.to(gpu_device), scale)
    for b, n in enumerate((333, 20)):
        check(pages, out, b, range(n), float(np.float32(scale)))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_query_that_is_not_finite(dtype, bad, gpu_device):
    pages = Fp4Pages([60], 8, 2, 128, 16, dtype, gpu_device)
    pages.q[0, 2, 70] = bad
    for scale in (0.1, 0.0, -2.0):
        out = span.paged_decode_attn_fp4(pages.q.to(gpu_device), *pages.cache(), pages.ctx.to(gpu_device), scale)
        assert out[0, 2].isnan().all() and not out[0, [0, 1, 3, 4, 5, 6, 7]].isnan().any()


def test_scores_far_apart(gpu_device):
    """The largest score moves on from slice to slice: weights that are nothing beside it are nothing, and large ones close together are weighed evenly."""
    pages = Fp4Pages([2000], 2, 1, 64, 16, "f32", gpu_device)
    pages.q *= 60
    out = span.paged_decode_attn_fp4(pages.q.to(gpu_device), *pages.cache(), pages.ctx.to(gpu_device), 1.0)
    want, bound = pages.attend(0, range(2000), 1.0)
    assert np.all(np.abs(out[0].cpu().double().numpy() - want) <= bound)
    assert bound.max() < 0.05 * np.abs(want).max()


def test_same_bits_again(gpu_device):
    """Slices are joined in a fixed order."""
    pages = Fp4Pages([5000, 3000, 17], 8, 4, 128, 64, "bf16", gpu_device)
    call = span.prepare_paged_decode_attn_fp4(pages.q.to(gpu_device), *pages.cache(), pages.ctx.to(gpu_device), 0.1)
    first = call().clone()
    for _ in range(200):
        assert torch.equal(call(), first)
