"""Rotated appends into pages of the storage type and of 4-bit values, and rows read back.  V, codes and exponents have to be equal; turned values are off by their roundings."""
import numpy as np
import pytest
import torch

import paper_2404_09336_amd as span
from paged_more_reference import from_fp4, place, rotation_table, to_fp4, turned, write_fp4
from paged_reference import DTYPES, Pages

pytestmark = pytest.mark.gpu

LENS = [5, 16, 17, 100, 64, 1, 90, 3]
MANY_LENS, MANY = [5, 200, 170, 33, 260, 1, 90, 3], [5, 187, 170, 33, 155, 1, 0, 7]  # more tokens than a step's: the kernels for those take longer chunks
NEW = {"one": [1] * 8, "some": [5, 0, 1, 70, 33, 1, 20, 7]}  # (the last has 7 new tokens at 3 positions)


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


class Rows:
    """New rows of the sequences above, some of nobody's, and where each of them goes: (row, sequence, slot, true position)."""

    def __init__(self, new, heads, kv_heads, head_dim, dtype, device, seed=0, ahead=0, lens=LENS):
        self.pages = Pages(lens, heads, kv_heads, head_dim, 16, dtype, device, seed=seed)
        self.pages.table[min(6, len(lens) - 1), -1] = -1
        if len(lens) > 4:
            self.pages.table[4, 3] = self.pages.K.shape[0]
        t = NEW[new] if isinstance(new, str) else new
        spare = 0 if new == "one" else 4
        total = sum(t) + spare
        g = self.pages.generator
        self.k, self.v, self.q = (torch.randn((total, n, head_dim), generator=g).to(DTYPES[dtype]) for n in (kv_heads, kv_heads, heads))
        self.off = None if new == "one" else torch.from_numpy(np.cumsum([0] + t).astype(np.int32))
        self.seen = torch.tensor([n + ahead * (b + 1) for b, n in enumerate(lens)], dtype=torch.int32)
        at = np.cumsum([0] + t)
        self.tokens = [(int(at[b]) + j, b, lens[b] - t[b] + j, int(self.seen[b]) - t[b] + j) for b in range(len(lens)) for j in range(t[b])]

    def slot(self, b, p):
        """(page, row) or None."""
        if not 0 <= p < self.pages.capacity:
            return None
        page = int(self.pages.table[b, p // 16])
        return (page, p % 16) if 0 <= page < self.pages.K.shape[0] else None

    def on(self, device, *names):
        return [None if getattr(self, n) is None else getattr(self, n).to(device) for n in names]


def within(got, want, size, dtype):
    """fp32 products and sum (half a step of one product, of the sum), then half a step of the type (of fp16's least numbers: 2^-25)."""
    got = got.double().numpy()
    eps = torch.finfo(DTYPES[dtype]).eps / 2 if dtype != "f32" else 0.0
    assert np.array_equal(np.isnan(got), np.isnan(want))
    bound = eps * np.abs(want) * (1 + 2.0 ** -20) + 2.0 ** -23 * size + (2.0 ** -25 if dtype == "f16" else 1e-37)
    assert np.all((np.abs(got - want) <= bound) | np.isnan(want))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads,kv_heads,head_dim", [(2, 1, 64), (9, 3, 128), (40, 40, 64)])
@pytest.mark.parametrize("channels,paired", [(64, False), (64, True), (16, False), (48, True), (48, False)])
@pytest.mark.parametrize("new", ["one", "some"])
def test_rotary(dtype, heads, kv_heads, head_dim, channels, paired, new, gpu_device):
    check_rotary(Rows(new, heads, kv_heads, head_dim, dtype, gpu_device, seed=channels, ahead=30), dtype, kv_heads, channels, paired, gpu_device)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads,kv_heads,head_dim", [(2, 1, 64), (9, 3, 128), (11, 11, 64)])
@pytest.mark.parametrize("channels,paired", [(64, False), (64, True), (16, False), (48, True)])
def test_rotary_of_many_tokens(dtype, heads, kv_heads, head_dim, channels, paired, gpu_device):
    check_rotary(Rows(MANY, heads, kv_heads, head_dim, dtype, gpu_device, seed=channels, ahead=30, lens=MANY_LENS), dtype, kv_heads, channels, paired, gpu_device)


def check_rotary(r, dtype, kv_heads, channels, paired, gpu_device):
    angles = rotation_table(500, channels)
    K, V, table, ctx = r.pages.to("K", "V", "table", "ctx")
    k, v, q, off, seen = r.on(gpu_device, "k", "v", "q", "off", "seen")
    positions = torch.full((8, kv_heads, r.pages.capacity), -9, dtype=torch.int32)
    pos = positions.to(gpu_device)
    q_out = torch.full_like(q, 7.0)
    span.paged_append_rotary(k, v, K, V, table, ctx, angles.to(gpu_device), off, paired=paired, q=q, q_out=q_out, positions=pos, seen=seen)
    want_k, size_k = r.pages.K.double().numpy(), np.zeros(r.pages.K.shape)
    written = torch.zeros(r.pages.K.shape[:3], dtype=torch.bool)
    want_q, size_q = np.full(r.q.shape, 7.0), np.zeros(r.q.shape)
    for row, b, p, position in r.tokens:
        want_q[row], size_q[row] = turned(r.q[row].double().numpy(), angles, position, paired)
        if 0 <= p < r.pages.capacity:
            positions[b, :, p] = position
        if r.slot(b, p):
            page, at = r.slot(b, p)
            want_k[page, :, at], size_k[page, :, at] = turned(r.k[row].double().numpy(), angles, position, paired)
            r.pages.V[page, :, at] = r.v[row]
            written[page, :, at] = True
    assert same(V.cpu(), r.pages.V) and torch.equal(pos.cpu(), positions)
    assert same(K.cpu()[~written], r.pages.K[~written])
    mask = written.numpy()
    within(K.cpu()[written], want_k[mask], size_k[mask], dtype)
    assert torch.equal(K.cpu()[written][:, channels:], torch.from_numpy(want_k[mask])[:, channels:].to(DTYPES[dtype]))
    within(q_out.cpu(), want_q, size_q, dtype)
    assert torch.equal(q_out.cpu()[..., channels:], torch.from_numpy(want_q)[..., channels:].to(DTYPES[dtype]))


def test_rotary_without_q_and_in_place(gpu_device):
    r = Rows("some", 4, 2, 64, "f16", gpu_device)
    angles = rotation_table(200, 64).to(gpu_device)
    k, v, q, off = r.on(gpu_device, "k", "v", "q", "off")
    pools = [r.pages.to("K", "V") for _ in range(3)]
    table, ctx = r.pages.to("table", "ctx")
    kept = q.clone()
    _, _, out = span.paged_append_rotary(k, v, *pools[0], table, ctx, angles, off, q=q)
    assert same(q, kept)
    both = span.paged_append_rotary(k, v, *pools[1], table, ctx, angles, off)
    assert len(both) == 2 and same(pools[0][0], pools[1][0])
    span.paged_append_rotary(k, v, *pools[2], table, ctx, angles, off, q=q, q_out=q)
    rows = [row for row, *_ in r.tokens]
    assert same(q[rows], out[rows]) and same(pools[0][0], pools[2][0]) and same(q[len(rows):], kept[len(rows):])  # (nobody's rows are left alone)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_positions_without_angles(dtype, gpu_device):
    """The turned channels become NaN, K's and q's; the others, V and everybody else stay."""
    r = Rows("one", 4, 2, 128, dtype, gpu_device)
    angles = rotation_table(64, 32)
    K, V, table, ctx = r.pages.to("K", "V", "table", "ctx")
    k, v, q = r.on(gpu_device, "k", "v", "q")
    seen = torch.tensor([64, 65, 0, -5, 1, 2, 1 << 30, 4], dtype=torch.int32)  # positions 63, 64, -1, -6, 0, 1, far, 3
    out = span.paged_append_rotary(k, v, K, V, table, ctx, angles.to(gpu_device), q=q, seen=seen.to(gpu_device))[2].cpu()
    missing = [1, 2, 3, 6]
    assert out[missing][..., :32].isnan().all() and not out[[0, 4, 5, 7]].isnan().any()
    assert same(out[..., 32:], r.q[..., 32:])
    for b in (1, 2, 3):
        page, at = r.slot(b, LENS[b] - 1)
        assert K[page, :, at, :32].isnan().all() and same(K[page, :, at, 32:].cpu(), r.k[b, :, 32:]) and same(V[page, :, at].cpu(), r.v[b])


def test_a_full_table_drops_rows_and_turns_their_queries(gpu_device):
    r = Rows([3, 2], 4, 2, 64, "f32", gpu_device, lens=[16, 16])
    angles = rotation_table(40, 64)
    K, V, table = r.pages.to("K", "V", "table")
    r.pages.table[:] = table.cpu()
    ctx = torch.tensor([18, 20], dtype=torch.int32)  # slots 15, 16, 17 and 18, 19 of 16
    k, v, q, off = r.on(gpu_device, "k", "v", "q", "off")
    out = span.paged_append_rotary(k, v, K, V, table, ctx.to(gpu_device), angles.to(gpu_device), off, q=q)[2].cpu()
    for row, position in enumerate((15, 16, 17, 18, 19)):
        want, size = turned(r.q[row].double().numpy(), angles, position, False)
        within(out[row], want, size, "f32")
    want = r.pages.K.clone()
    if 0 <= int(table[0, 0]) < K.shape[0]:
        page = int(table[0, 0])
        y, size = turned(r.k[0].double().numpy(), angles, 15, False)
        within(K[page, :, 15].cpu(), y, size, "f32")
        want[page, :, 15] = K[page, :, 15].cpu()
    assert same(K.cpu(), want)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads,kv_heads,head_dim", [(2, 1, 64), (9, 3, 128), (40, 40, 64)])
@pytest.mark.parametrize("channels,paired", [(0, False), (64, False), (64, True), (48, False), (16, True)])
@pytest.mark.parametrize("new", ["one", "some"])
def test_fp4(dtype, heads, kv_heads, head_dim, channels, paired, new, gpu_device):
    """Every byte of the pools, the rows read back, and q."""
    check_fp4(Rows(new, heads, kv_heads, head_dim, dtype, gpu_device, seed=channels + 1, ahead=30), dtype, kv_heads, head_dim, channels, paired, gpu_device)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads,kv_heads,head_dim", [(2, 1, 64), (9, 3, 128), (11, 11, 64), (18, 18, 128)])
@pytest.mark.parametrize("channels,paired", [(0, False), (64, False), (64, True), (48, False), (16, True)])
def test_fp4_of_many_tokens(dtype, heads, kv_heads, head_dim, channels, paired, gpu_device):
    r = Rows(MANY, heads, kv_heads, head_dim, dtype, gpu_device, seed=channels + 1, ahead=30, lens=MANY_LENS)
    check_fp4(r, dtype, kv_heads, head_dim, channels, paired, gpu_device)


def check_fp4(r, dtype, kv_heads, head_dim, channels, paired, gpu_device):
    scale = 2.0 ** torch.randint(-8, 9, (*r.k.shape[:2], head_dim // 32), generator=r.pages.generator).repeat_interleave(32, -1)
    r.k, r.v = (r.k * scale).to(r.k.dtype), (r.v * scale).to(r.k.dtype)
    angles = rotation_table(500, channels) if channels else None
    N, row_bytes = r.pages.K.shape[0], head_dim // 2 + head_dim // 32
    g = torch.Generator().manual_seed(3)
    pools = [torch.randint(0, 256, (N, kv_heads, 16, row_bytes), generator=g).to(torch.uint8) for _ in range(2)]
    K, V = (p.to(gpu_device) for p in pools)
    table, ctx = r.pages.to("table", "ctx")
    k, v, q, off, seen = r.on(gpu_device, "k", "v", "q", "off", "seen")
    k_rows, v_rows = torch.full_like(k, 5.0), torch.full_like(v, 6.0)
    got = span.paged_append_fp4(k, v, K, V, table, ctx, off, rotation=None if angles is None else angles.to(gpu_device), paired=paired, q=q if channels else None, seen=seen)
    span.paged_read_fp4(K, V, table, ctx, off, k_rows=k_rows, v_rows=v_rows)
    want = [p.reshape(N, kv_heads, -1).numpy().copy() for p in pools]
    want_rows = [np.full(r.k.shape, 5.0), np.full(r.k.shape, 6.0)]
    for row, b, p, position in r.tokens:
        kx = r.k[row].double().numpy()
        if channels:
            kx = turned(kx, angles, position, paired)[0]
            w, size = turned(r.q[row].double().numpy(), angles, position, paired)
            within(got[2][row].cpu(), w, size, dtype)
        if r.slot(b, p):
            page, at = r.slot(b, p)
            for i, x in enumerate((kx, r.v[row].double().numpy())):
                code, byte = to_fp4(x)
                for h in range(kv_heads):
                    write_fp4(want[i][page, h], 16, head_dim, at, i == 1, code[h], byte[h])
                want_rows[i][row] = from_fp4(code, byte)
    for got_pool, w in zip((K, V), want):
        assert np.array_equal(got_pool.cpu().reshape(N, kv_heads, -1).numpy(), w)
    for got_rows, w in zip((k_rows, v_rows), want_rows):
        assert np.array_equal(got_rows.cpu().double().numpy(), w)  # (all of them numbers that the type holds)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("head_dim", [64, 128])
def test_fp4_extremes(dtype, head_dim, gpu_device):
    """The largest and the smallest numbers of the type, borders between values, zeros of both signs, NaN and infinity in one block: its neighbours stay."""
    info = torch.finfo(DTYPES[dtype])
    tiny = {"f16": 2.0 ** -24, "bf16": 2.0 ** -133, "f32": 2.0 ** -149}[dtype]
    rows = [torch.full((head_dim,), info.max), torch.full((head_dim,), tiny), torch.full((head_dim,), info.tiny), torch.zeros(head_dim), torch.full((head_dim,), -0.0)]
    edge = torch.zeros(head_dim)
    edge[:16] = torch.tensor([7, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5, -7])
    rows += [edge, edge * 2.0 ** -10, edge * 3]
    near = edge.to(DTYPES[dtype]).clone()
    near = torch.nextafter(near, torch.full_like(near, 100.0)).float()
    rows += [near, torch.nextafter(edge.to(DTYPES[dtype]), torch.zeros(head_dim, dtype=DTYPES[dtype])).float()]
    for bad in (float("nan"), float("inf"), -float("inf")):
        x = torch.randn(head_dim, generator=torch.Generator().manual_seed(1))
        x[5] = bad
        rows.append(x)
    if dtype != "f16":
        rows += [torch.full((head_dim,), 2.9e38), torch.full((head_dim,), 3.0e38), edge * 2.0 ** -126, edge * 2.0 ** -128, edge * 2.0 ** 124]
    x = torch.stack(rows).to(DTYPES[dtype])[:, None]  # [tokens, 1, head_dim]
    n = x.shape[0]
    K, V = (torch.full((3, 1, 16, head_dim // 2 + head_dim // 32), 0xA5, dtype=torch.uint8, device=gpu_device) for _ in range(2))
    table, ctx = torch.tensor([[2, 0]], dtype=torch.int32, device=gpu_device), torch.tensor([n], dtype=torch.int32, device=gpu_device)
    off = torch.tensor([0, n], dtype=torch.int32, device=gpu_device)
    xg = x.to(gpu_device)
    span.paged_append_fp4(xg, xg, K, V, table, ctx, off)
    out = [torch.zeros_like(xg) for _ in range(2)]
    span.paged_read_fp4(K, V, table, ctx, off, k_rows=out[0], v_rows=out[1])
    code, byte = to_fp4(x[:, 0].double().numpy())
    want = torch.from_numpy(from_fp4(code, byte))
    for is_v, (pool, rows_out) in enumerate(((K, out[0]), (V, out[1]))):
        flat = pool.cpu().reshape(3, -1).numpy()
        for t in range(n):
            page = [2, 0][t // 16]
            codes, exps = place(16, head_dim, t % 16, is_v == 1)
            assert np.array_equal(flat[page][exps], byte[t]), t
            keep = np.repeat(byte[t] != 255, 16)  # (what a block that is NaN holds beside its exponent means nothing)
            assert np.array_equal(flat[page][codes][keep], (code[t][0::2] | (code[t][1::2] << 4))[keep]), t
        got = rows_out[:, 0].cpu()
        assert torch.equal(got.isnan(), want.isnan())
        assert bool((got == want.to(DTYPES[dtype]))[~want.isnan()].all())  # (values that the type does not hold: infinite on both sides)


def test_turned_values_next_to_borders(gpu_device):
    """One rounding, as if K had been turned exactly: angles and rows whose turned values are a few units of the 64-bit sum from a border, where a rounding to fp32 ahead of it would
    put them on the border."""
    D, n = 64, 64
    angles = torch.zeros((n, 32))
    x = torch.zeros((n, 1, D))
    for t in range(n):
        # channel 0: x0 c - x16 s = border + (+-) tiny;  c = 1, s = 2^-20, x16 = -+2^-10
        border = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0][t % 7]
        x[t, 0, 0], x[t, 0, 16], x[t, 0, 1] = border, (-1.0) ** (t // 7) * 2.0 ** -10, 6.0
        angles[t, :16], angles[t, 16:] = 1.0, 2.0 ** -20
    K, V = (span.fp4_pages(5, 1, 16, D, gpu_device) for _ in range(2))
    table = torch.arange(4, dtype=torch.int32, device=gpu_device)[None].contiguous()
    ctx, off = torch.tensor([n], dtype=torch.int32, device=gpu_device), torch.tensor([0, n], dtype=torch.int32, device=gpu_device)
    xg = x.to(gpu_device)
    span.paged_append_fp4(xg, xg, K, V, table, ctx, off, rotation=angles.to(gpu_device))
    rows = [torch.zeros_like(xg) for _ in range(2)]
    span.paged_read_fp4(K, V, table, ctx, off, k_rows=rows[0], v_rows=rows[1])
    differ = 0
    for t in range(n):
        y = turned(x[t].double().numpy(), angles, t, False)[0]
        want = from_fp4(*to_fp4(y))
        assert np.array_equal(rows[0][t].cpu().double().numpy(), want), t
        differ += not np.array_equal(want, from_fp4(*to_fp4(y.astype(np.float32))))
    assert differ >= 16  # (rounded to fp32 first, as many rows would be others)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads,kv_heads,head_dim", [(2, 1, 64), (9, 3, 128)])
@pytest.mark.parametrize("new", ["some", MANY])
@pytest.mark.parametrize("in_place", [False, True])
def test_queries_without_rotation(dtype, heads, kv_heads, head_dim, new, in_place, gpu_device):
    """They pass through, those of dropped rows too; nobody's are left alone; the pools are those of a call without q."""
    r = Rows(new, heads, kv_heads, head_dim, dtype, gpu_device, lens=MANY_LENS if new is MANY else LENS)
    table, ctx = r.pages.to("table", "ctx")
    k, v, q, off = r.on(gpu_device, "k", "v", "q", "off")
    q_out = q if in_place else torch.full_like(q, 7.0)
    pools = [[span.fp4_pages(r.pages.K.shape[0], kv_heads, 16, head_dim, gpu_device) for _ in range(2)] for _ in range(2)]
    span.paged_append_fp4(k, v, *pools[0], table, ctx, off)
    got = span.paged_append_fp4(k, v, *pools[1], table, ctx, off, q=q, q_out=q_out)
    assert len(got) == 3 and got[2] is q_out and all(same(a, b) for a, b in zip(*pools))
    rows = [row for row, *_ in r.tokens]
    want = r.q.clone() if in_place else torch.full_like(r.q, 7.0)
    want[rows] = r.q[rows]
    assert same(q_out.cpu(), want)


@pytest.mark.parametrize("paired", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_turned_values_next_to_borders_of_many_tokens(dtype, paired, gpu_device):
    """Values that are a few units of fp32 and less from a border, or on it, between others of every size; blocks whose largest value is next to where the exponent changes."""
    D, n, C = 128, 640, 64
    g = torch.Generator().manual_seed(8)
    x = torch.randn((n, 2, D), generator=g) * 2.0 ** torch.randint(-20, 21, (n, 2, 1), generator=g)
    angles = rotation_table(n, C)
    one = [2 * i for i in range(32)] if paired else list(range(32))
    two = [2 * i + 1 for i in range(32)] if paired else list(range(32, 64))
    for t in range(0, n, 2):  # angle 0 and almost: x cos - x' sin = border + j tiny
        angles[t, :32], angles[t, 32:] = 1.0, 2.0 ** -18
        for i in range(32):
            x[t, 0, one[i]] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0][(t // 2 + i) % 8] * (1 if i % 3 else -1)
            x[t, 0, two[i]] = float(torch.randint(-3, 4, (1,), generator=g)) * 2.0 ** -(6 + t % 16)
    x = x.to(DTYPES[dtype])
    K, V = (span.fp4_pages(40, 2, 16, D, gpu_device) for _ in range(2))
    table = torch.arange(40, dtype=torch.int32, device=gpu_device)[None].contiguous()
    ctx, off = torch.tensor([n], dtype=torch.int32, device=gpu_device), torch.tensor([0, n], dtype=torch.int32, device=gpu_device)
    xg = x.to(gpu_device)
    span.paged_append_fp4(xg, xg, K, V, table, ctx, off, rotation=angles.to(gpu_device), paired=paired)
    flat = K.cpu().reshape(40, 2, -1).numpy()
    for t in range(n):
        code, byte = to_fp4(turned(x[t].double().numpy(), angles, t, paired)[0])
        codes, exps = place(16, D, t % 16, False)
        for h in range(2):
            assert np.array_equal(flat[t // 16, h][exps], byte[h]), (t, h)
            assert np.array_equal(flat[t // 16, h][codes], code[h][0::2] | (code[h][1::2] << 4)), (t, h)


@pytest.mark.parametrize("exponent", [-126, -125, -124, -110, 0, 125])
def test_turned_values_next_to_borders_of_any_size(exponent, gpu_device):
    """The same in blocks whose values, or borders, fp32 holds with fewer bits than 24 or not at all."""
    D, n = 64, 16
    angles, x = torch.zeros((n, 32)), torch.zeros((n, 1, D))
    for t in range(n):
        border = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0][t % 7]
        x[t, 0, 0], x[t, 0, 16], x[t, 0, 1] = border, (-1.0) ** (t // 7) * 2.0 ** -10, 6.0
        angles[t, :16], angles[t, 16:] = 1.0, 2.0 ** -20
    x = (x.double() * 2.0 ** exponent).float()  # (exact: 2^-10 * 2^-126 is a multiple of 2^-149)
    K, V = (span.fp4_pages(1, 1, 16, D, gpu_device) for _ in range(2))
    table = torch.zeros((1, 1), dtype=torch.int32, device=gpu_device)
    ctx, off = torch.tensor([n], dtype=torch.int32, device=gpu_device), torch.tensor([0, n], dtype=torch.int32, device=gpu_device)
    xg = x.to(gpu_device)
    span.paged_append_fp4(xg, xg, K, V, table, ctx, off, rotation=angles.to(gpu_device))
    flat = K.cpu().reshape(-1).numpy()
    for t in range(n):
        code, byte = to_fp4(turned(x[t].double().numpy(), angles, t, False)[0])
        codes, exps = place(16, D, t, False)
        assert np.array_equal(flat[exps], byte[0]) and byte[0][0] == exponent + 127, t
        assert np.array_equal(flat[codes], code[0][0::2] | (code[0][1::2] << 4)), t


def test_fp4_beyond_four_gib(gpu_device):
    """Pages whose bytes lie past 32 bits."""
    N, KV, P, D = 66000, 8, 128, 128
    K, V = (torch.empty((N, KV, P, D // 2 + D // 32), dtype=torch.uint8, device=gpu_device) for _ in range(2))
    assert K.numel() > 1 << 32
    table = torch.tensor([[N - 1], [N // 2 + 12345]], dtype=torch.int32, device=gpu_device)
    for page in table.flatten().tolist():
        K[page], V[page] = 0, 0
    ctx = torch.tensor([128, 100], dtype=torch.int32, device=gpu_device)
    off = torch.tensor([0, 128, 228], dtype=torch.int32, device=gpu_device)
    x = torch.randn((228, KV, D), generator=torch.Generator().manual_seed(0)).to(torch.bfloat16).to(gpu_device)
    span.paged_append_fp4(x, -x, K, V, table, ctx, off)
    rows = [torch.zeros_like(x) for _ in range(2)]
    span.paged_read_fp4(K, V, table, ctx, off, k_rows=rows[0], v_rows=rows[1])
    want = torch.from_numpy(from_fp4(*to_fp4(x.cpu().double().numpy())))
    assert torch.equal(rows[0].cpu().double(), want) and torch.equal(rows[1].cpu().double(), -want)
    q = torch.randn((2, 16, D), generator=torch.Generator().manual_seed(1)).to(gpu_device)
    out = span.paged_decode_attn_fp4(q, K, V, table, ctx, 0.1).cpu().double()
    for b in range(2):
        k = want[[slice(0, 128), slice(128, 228)][b]].transpose(0, 1)
        w = torch.softmax(q[b].cpu().double().reshape(KV, 2, D) @ k.transpose(1, 2).contiguous() * 0.1, -1)
        assert float((out[b].reshape(KV, 2, D) + w @ k).abs().max()) < 1e-4
