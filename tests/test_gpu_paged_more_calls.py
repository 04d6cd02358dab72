"""Turned and 4-bit appends, attention over 4-bit pages, page selection and attention over chosen pages as programs call them: together over the life of a cache, refusals of the binding,
streams, calls side by side, captured steps, shared workspaces."""
import numpy as np
import pytest
import torch

import paper_2404_09336_amd as span
from paged_more_reference import from_fp4, place, read_fp4, rotation_table, select, to_fp4, turned
from paged_reference import Pages, attend

pytestmark = pytest.mark.gpu

B, H, KV, D, P = 5, 8, 2, 64, 16
LENS = [300, 61, 60, 7, 190]


def same(a, b):
    return all(torch.equal(x.cpu().contiguous().view(torch.uint8), y.cpu().contiguous().view(torch.uint8)) for x, y in zip(a, b))


class Setting:
    def __init__(self, device, seed=0):
        pages = Pages(LENS, H, KV, D, P, "f16", device, seed=seed, table_pages=20)
        self.K, self.V, self.table, self.ctx = pages.to("K", "V", "table", "ctx")
        g = pages.generator
        N = self.K.shape[0]
        self.q = pages.q.to(device)
        self.new = [torch.randn((B, KV, D), generator=g).half().to(device) for _ in range(2)]
        self.prompt = [torch.randn((B * 3, n, D), generator=g).half().to(device) for n in (KV, KV, H)]
        self.offsets = torch.arange(0, 3 * B + 1, 3, dtype=torch.int32, device=device)
        self.rotation = rotation_table(400, 48).to(device)
        self.seen = self.ctx + 50
        self.positions = torch.full((B, KV, 20 * P), -1, dtype=torch.int32, device=device)
        self.bounds = torch.zeros((N, KV, 2, D), dtype=torch.float16, device=device)
        self.since = torch.zeros(B, dtype=torch.int32, device=device)
        self.K4, self.V4 = (torch.randint(0, 128, (N, KV, P, D // 2 + D // 32), generator=g).to(torch.uint8).to(device) for _ in range(2))
        self.spans = [torch.tensor(x, dtype=torch.int32, device=device) for x in
                      ([0, 2, 3, 4, 5, 6], [0, 250, 10, 0, 3, 100], [20, 300, 61, 60, 7, 130])]
        self.selected = torch.tensor([[[0, 3, -1]] * KV, [[3, 1, 0]] * KV, [[1, 2, 3]] * KV, [[0, -1, -1]] * KV, [[2, 7, 11]] * KV], dtype=torch.int32, device=device)
        self.rows = [torch.zeros((B * 3, KV, D), dtype=torch.float16, device=device) for _ in range(2)]

    def rotary(self, **kw):
        return span.paged_append_rotary(*self.prompt[:2], self.K, self.V, self.table, self.ctx, self.rotation, self.offsets, q=self.prompt[2], seen=self.seen,
                                        positions=self.positions, **kw)

    def append(self, **kw):
        return span.paged_append_fp4(*self.prompt[:2], self.K4, self.V4, self.table, self.ctx, self.offsets, rotation=self.rotation, q=self.prompt[2], seen=self.seen, **kw)

    def read(self, **kw):
        return span.paged_read_fp4(self.K4, self.V4, self.table, self.ctx, self.offsets, k_rows=self.rows[0], v_rows=self.rows[1], **kw)

    def decode(self, **kw):
        return span.paged_decode_attn_fp4(self.q, self.K4, self.V4, self.table, self.ctx, 0.125, **kw)

    def decode_spans(self, **kw):
        return span.paged_span_decode_attn_fp4(self.q, self.K4, self.V4, self.table, *self.spans, 0.125, **kw)

    def select(self, **kw):
        return span.paged_select(self.q, self.K, self.bounds, self.table, self.ctx, 6, sinks=4, recent=20, since=self.since, **kw)

    def chosen(self, **kw):
        return span.paged_selected_decode_attn(self.q, self.K, self.V, self.table, self.ctx, self.selected, 0.125, **kw)


def misaligned(t):
    """The same values one element (of less than 16 bytes) off."""
    store = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
    store[1:] = t.reshape(-1)
    return store[1:].view(t.shape)


@pytest.mark.parametrize("what", ["K", "V", "K4", "V4", "table", "ctx", "q", "new", "rotation", "offsets", "seen", "positions", "bounds", "since", "selected", "rows", "spans"])
def test_refused_tensors(what, gpu_device):
    """Another type, another shape, not contiguous, not aligned, not on the GPU: each tensor, in the calls that take it, before anything is launched."""
    s = Setting(gpu_device)
    calls = {"K": [s.rotary, s.select, s.chosen], "V": [s.rotary, s.chosen], "K4": [s.append, s.read, s.decode, s.decode_spans], "V4": [s.append, s.read, s.decode],
             "table": [s.rotary, s.append, s.read, s.decode, s.select, s.chosen], "ctx": [s.rotary, s.append, s.read, s.decode, s.select, s.chosen],
             "q": [s.decode, s.select, s.chosen], "new": [s.rotary, s.append], "rotation": [s.rotary, s.append], "offsets": [s.rotary, s.append, s.read],
             "seen": [s.rotary, s.append], "positions": [s.rotary], "bounds": [s.select], "since": [s.select], "selected": [s.chosen], "rows": [s.read], "spans": [s.decode_spans]}[what]
    before = {n: getattr(s, n).clone() for n in ("K", "V", "K4", "V4", "bounds", "positions")}
    name = "prompt" if what == "new" else what
    good = getattr(s, name)
    at = {"new": 1, "rows": 1, "spans": 1}.get(what)
    one = good if at is None else good[at]
    other_shape = lambda t: torch.cat((t, t), dim=0 if what == "table" else t.dim() - 1)[..., :-1].contiguous()  # noqa: E731
    doubled = lambda t: torch.stack((t, t), dim=-1)[..., 0]  # noqa: E731
    bad = [lambda t: t.double() if t.is_floating_point() else t.long(), doubled, misaligned, lambda t: t.cpu()]
    if what != "selected":  # (a list of another length is another budget)
        bad.append(other_shape)
    for f in bad:
        setattr(s, name, f(good) if at is None else [*good[:at], f(good[at]), *good[at + 1:]])
        for call in calls:
            with pytest.raises((ValueError, TypeError, span.SpanAttnError)):  # (TypeError: a type that no call takes)
                call()
    assert not doubled(one).is_contiguous()
    setattr(s, name, good)
    assert same([getattr(s, n) for n in before], before.values())
    for call in calls:
        call()


def test_refused_arguments(gpu_device):
    s = Setting(gpu_device)
    half = s.prompt[2][:, :, :32].contiguous()
    calls = [lambda: span.paged_decode_attn_fp4(s.q.double(), s.K4, s.V4, s.table, s.ctx, 1.0), lambda: s.decode(window=-1), lambda: s.decode(sinks=1 << 31),
             lambda: span.paged_append_fp4(*s.new, s.K4, s.V4, s.table, s.ctx, q_out=s.q), lambda: span.paged_append_fp4(*s.new, s.K4, s.V4, s.table, s.ctx, s.offsets[:3]),
             lambda: span.paged_append_rotary(*s.new, s.K, s.V, s.table, s.ctx, None), lambda: span.paged_append_rotary(*s.new, s.K, s.V, s.table, s.ctx, s.rotation[:, :24].contiguous()),
             lambda: span.paged_append_rotary(*s.new, s.K, s.V, s.table, s.ctx, s.rotation, q_out=s.q), lambda: s.rotary(q_out=half), lambda: s.rotary(q_out=s.prompt[2].float()),
             lambda: span.paged_append_rotary(*s.prompt[:2], s.K, s.V, s.table, s.ctx, s.rotation), lambda: span.paged_read_fp4(s.K4, s.V4, s.table, s.ctx, k_rows=s.rows[0], v_rows=s.rows[1]),
             lambda: span.paged_select(s.q, s.K, s.bounds, s.table, s.ctx, 0), lambda: span.paged_select(s.q, s.K, s.bounds, s.table, s.ctx, 2, sinks=17),
             lambda: span.paged_select(s.q, s.K, s.bounds, s.table, s.ctx, 6, recent=-1), lambda: s.select(selected=s.selected), lambda: s.select(workspace=torch.zeros(64, dtype=torch.uint8, device=gpu_device)),
             lambda: span.paged_selected_decode_attn(s.q, s.K, s.V, s.table, s.ctx, s.selected[0], 1.0), lambda: s.chosen(out=torch.empty((B, H, D), dtype=torch.float16, device=gpu_device)),
             lambda: span.paged_selected_decode_attn(s.q, s.K, s.V, s.table, s.ctx, s.selected[:, :, :0].contiguous(), 1.0),
             lambda: span.paged_decode_attn_fp4(s.q, s.K4[..., :33].contiguous(), s.V4[..., :33].contiguous(), s.table, s.ctx, 1.0), lambda: span.paged_decode_attn_fp4(s.q, s.K, s.V, s.table, s.ctx, 1.0),
             lambda: span.paged_decode_attn(s.q, s.K4, s.V4, s.table, s.ctx, 1.0)]
    buffer = torch.zeros(2 * s.prompt[2].numel(), dtype=torch.float16, device=gpu_device)
    view = lambda at: buffer[at:at + s.prompt[2].numel()].view(s.prompt[2].shape)  # noqa: E731
    calls.append(lambda: span.paged_append_rotary(*s.prompt[:2], s.K, s.V, s.table, s.ctx, s.rotation, s.offsets, q=view(0), q_out=view(64)))  # overlaps
    for call in calls:
        with pytest.raises((ValueError, TypeError, span.SpanAttnError)):
            call()


def results(s, **kw):
    """All operators; the caches are the setting's own."""
    out = [s.rotary(**kw)[2], s.append(**kw)[2], *s.read(**kw), s.decode(**kw), s.decode_spans(**kw), s.select(**kw), s.chosen(**kw)]
    return [*out, s.K, s.V, s.K4, s.V4, s.bounds, s.positions]


def test_another_stream_while_the_current_one_is_busy(gpu_device):
    """New outputs and workspaces belong to the call's stream."""
    want = results(Setting(gpu_device))
    torch.cuda.synchronize()
    side = torch.cuda.Stream(device=gpu_device)
    s = Setting(gpu_device)
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    got = results(s, stream=side.cuda_stream)
    side.synchronize()
    torch.cuda.synchronize()
    assert same(got, want)
    s = Setting(gpu_device)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
        got = results(s, stream=0)
    torch.cuda.synchronize()
    assert same(got, want)


def test_two_at_once(gpu_device):
    """The same steps on two streams at once, each with caches and workspaces of its own."""
    want = [results(Setting(gpu_device, seed)) for seed in (0, 1)]
    for _ in range(5):
        both, streams = [Setting(gpu_device, seed) for seed in (0, 1)], [torch.cuda.Stream(device=gpu_device) for _ in range(2)]
        torch.cuda.synchronize()
        got = [results(s, stream=x.cuda_stream) for s, x in zip(both, streams)]
        torch.cuda.synchronize()
        assert same(got[0], want[0]) and same(got[1], want[1])


def test_one_workspace_for_all(gpu_device):
    """Every call leaves the counters zero: calls that follow one another share a workspace, initialised once; calls that are cut into slices and into chunks among them."""
    lens = [16 * 900, 16 * 700 + 3]
    pages = Pages(lens, 4, 2, 64, 16, "bf16", gpu_device)
    K, V, table, ctx = pages.to("K", "V", "table", "ctx")
    K4, V4 = (torch.randint(0, 128, (K.shape[0], 2, 16, 34), generator=pages.generator).to(torch.uint8).to(gpu_device) for _ in range(2))
    q = pages.q.to(gpu_device)
    shared = torch.empty(1 << 24, dtype=torch.uint8, device=gpu_device)
    zero = torch.zeros(2, dtype=torch.int32, device=gpu_device)

    def steps(**kw):
        bounds = torch.zeros((K.shape[0], 2, 2, 64), dtype=torch.bfloat16, device=gpu_device)
        picked = span.paged_select(q, K, bounds, table, ctx, 200, since=zero, **kw)
        return [picked, span.paged_selected_decode_attn(q, K, V, table, ctx, picked, 0.1, **kw), span.paged_decode_attn_fp4(q, K4, V4, table, ctx, 0.1, **kw),
                span.paged_decode_attn(q, K, V, table, ctx, 0.1, **kw)]

    want = steps()
    call = span.prepare_paged_decode_attn(q, K, V, table, ctx, 0.1, workspace=shared)  # (for its descriptor)
    span.paged_workspace_init(call.desc)
    for _ in range(20):
        assert same(steps(workspace=shared), want)
    assert not shared[:4 * 2 * 3].any()  # tickets of the pairs and the sequences


def test_a_life_of_a_chosen_cache(gpu_device):
    """A prompt goes in turned and attends; then every step, one captured graph: rows go in turned, pages are bounded and chosen, the token attends them.  The plain form follows."""
    lens, H, KV, D, P, budget, cap = [150, 20], 4, 2, 64, 16, 5, 13
    pages = Pages([0, 0], H, KV, D, P, "f32", gpu_device, seed=3, table_pages=cap)
    K, V, table = pages.to("K", "V", "table")
    g = pages.generator
    angles = rotation_table(400, 64)
    rotation = angles.to(gpu_device)
    ctx = torch.tensor(lens, dtype=torch.int32, device=gpu_device)
    total = sum(lens)
    prompt = [torch.randn((total, n, D), generator=g) for n in (KV, KV, H)]
    off = torch.tensor([0, lens[0], total], dtype=torch.int32, device=gpu_device)
    k, v, q = (x.to(gpu_device) for x in prompt)
    _, _, q_turned = span.paged_append_rotary(k, v, K, V, table, ctx, rotation, off, q=q)
    out = span.paged_prompt_attn(q_turned, K, V, table, ctx, off, D ** -0.5).cpu()
    keys, values = [[] for _ in lens], [[] for _ in lens]  # what the caches hold, in 64 bits
    row = 0
    for b, n in enumerate(lens):
        for p in range(n):
            keys[b].append(turned(prompt[0][row].double().numpy(), angles, p, False)[0])
            values[b].append(prompt[1][row].double().numpy())
            if p in (0, n // 2, n - 1):
                check_attention(out[row], turned(prompt[2][row].double().numpy(), angles, p, False)[0], keys[b], values[b], [list(range(p + 1))] * KV, D ** -0.5)
            row += 1
    bounds = torch.zeros((K.shape[0], KV, 2, D), device=gpu_device)
    since = torch.zeros(2, dtype=torch.int32, device=gpu_device)
    k_new, v_new, q_new = (torch.zeros((2, n, D), device=gpu_device) for n in (KV, KV, H))
    side = torch.cuda.Stream(device=gpu_device)
    put = span.prepare_paged_append_rotary(k_new, v_new, K, V, table, ctx, rotation, q=q_new, q_out=q_new, stream=side.cuda_stream)
    choose = span.prepare_paged_select(q_new, K, bounds, table, ctx, budget, sinks=3, recent=10, since=since, stream=side.cuda_stream)
    look = span.prepare_paged_selected_decode_attn(q_new, K, V, table, ctx, choose.out, D ** -0.5, stream=side.cuda_stream)
    torch.cuda.synchronize()
    step = torch.cuda.CUDAGraph()
    with torch.cuda.graph(step, stream=side):
        ctx.add_(1)
        put()
        choose()
        look()
        since.copy_(ctx)  # all bounded now
    for t in range(45):
        new = [torch.randn(x.shape, generator=g) for x in (k_new, v_new, q_new)]
        for x, y in zip((k_new, v_new, q_new), new):
            x.copy_(y)
        torch.cuda.synchronize()
        step.replay()
        torch.cuda.synchronize()
        for b in range(2):
            n = lens[b] + t + 1
            keys[b].append(turned(new[0][b].double().numpy(), angles, n - 1, False)[0])
            values[b].append(new[1][b].double().numpy())
            qt = q_new[b].cpu().double().numpy()
            held = K[table[b].long()].cpu().double().numpy().transpose(1, 0, 2, 3).reshape(KV, -1, D)[:, :n]  # bounds are of what is held, roundings and all
            tops = [np.stack([np.stack((held[h, i:i + P].min(0), held[h, i:i + P].max(0))) for i in range(0, n, P)]) for h in range(KV)]
            lists = [select(qt.reshape(KV, H // KV, D)[h], tops[h], n, list(range(len(tops[h]))), P, budget, 3, 10) for h in range(KV)]
            assert choose.out[b].tolist() == lists
            check_attention(look.out[b].cpu(), turned(new[2][b].double().numpy(), angles, n - 1, False)[0], keys[b], values[b],
                            [[p for j in x if j >= 0 for p in range(j * P, min(j * P + P, n))] for x in lists], D ** -0.5)
    assert ctx.tolist() == [195, 65]


def check_attention(out, q, keys, values, positions, scale):
    KV = len(positions)
    G = q.shape[0] // KV
    for h in range(KV):
        k, v = (np.stack([x[p][h] for p in positions[h]]) for x in (keys, values))
        s = q[h * G:(h + 1) * G] @ k.T * scale
        w = np.exp(s - s.max(-1, keepdims=True))
        # fp32 roundings of turned rows, scores of some units, weights and sums: some 2^-20 of values of a few units
        assert np.abs(out[h * G:(h + 1) * G].double().numpy() - (w / w.sum(-1, keepdims=True)) @ v).max() <= 2e-5


def test_a_life_of_a_cache_in_4_bits(gpu_device):
    """Steps from a captured graph: rows go in turned and in 4 bits, the token attends them in a window with sinks; now and then a chunk of several tokens goes in eagerly, whose
    prompt attends a copy in the storage type that is read back.  What is attended is what the pages hold."""
    H, KV, D, P, cap, window, sinks = 4, 2, 64, 32, 5, 40, 3
    lens = [40, 1]
    g = torch.Generator().manual_seed(4)
    angles = rotation_table(400, 32)
    rotation = angles.to(gpu_device)
    N = 2 * cap + 1
    K, V = (span.fp4_pages(N, KV, P, D, gpu_device) for _ in range(2))
    table = torch.randperm(N, generator=g)[:2 * cap].reshape(2, cap).to(torch.int32).to(gpu_device)
    ctx = torch.tensor(lens, dtype=torch.int32, device=gpu_device)
    total = sum(lens)
    fresh = [torch.randn((total, KV, D), generator=g).to(torch.bfloat16).to(gpu_device) for _ in range(2)]
    span.paged_append_fp4(*fresh, K, V, table, ctx, torch.tensor([0, lens[0], total], dtype=torch.int32, device=gpu_device), rotation=rotation, paired=True)
    k_new, v_new, q_new = (torch.zeros((2, n, D), dtype=torch.bfloat16, device=gpu_device) for n in (KV, KV, H))
    side = torch.cuda.Stream(device=gpu_device)
    put = span.prepare_paged_append_fp4(k_new, v_new, K, V, table, ctx, rotation=rotation, paired=True, q=q_new, q_out=q_new, stream=side.cuda_stream)
    look = span.prepare_paged_decode_attn_fp4(q_new, K, V, table, ctx, D ** -0.5, window=window, sinks=sinks, stream=side.cuda_stream)
    torch.cuda.synchronize()
    step = torch.cuda.CUDAGraph()
    with torch.cuda.graph(step, stream=side):
        ctx.add_(1)
        put()
        look()

    def held(pool, b, is_v, n):
        return read_fp4(pool[table[b].long()].cpu().numpy(), is_v).transpose(1, 0, 2, 3).reshape(KV, -1, D)[:, :n]

    for t in range(30):
        if t % 10 == 9:  # three tokens of a prompt
            chunk = [torch.randn((6, n, D), generator=g).to(torch.bfloat16).to(gpu_device) for n in (KV, KV, H)]
            off = torch.tensor([0, 3, 6], dtype=torch.int32, device=gpu_device)
            ctx.add_(3)
            q = span.paged_append_fp4(*chunk[:2], K, V, table, ctx, off, rotation=rotation, paired=True, q=chunk[2])[2]
            counts = ctx.tolist()
            every = torch.tensor([0, counts[0], sum(counts)], dtype=torch.int32, device=gpu_device)
            rows = [torch.zeros((sum(counts), KV, D), dtype=torch.bfloat16, device=gpu_device) for _ in range(2)]
            span.paged_read_fp4(K, V, table, ctx, every, k_rows=rows[0], v_rows=rows[1])
            wide = [torch.zeros((N, KV, P, D), dtype=torch.bfloat16, device=gpu_device) for _ in range(2)]
            span.paged_append(*rows, *wide, table, ctx, every)
            out = span.paged_prompt_attn(q, *wide, table, ctx, off, D ** -0.5).cpu().double().numpy()
            for b in range(2):
                k, v = held(K, b, False, counts[b]), held(V, b, True, counts[b])
                assert np.array_equal(rows[0][every[b]:every[b + 1]].cpu().double().numpy().transpose(1, 0, 2), k)
                for i in range(3):
                    n = counts[b] - 2 + i
                    s = np.einsum("hgd,hnd->hgn", q[3 * b + i].cpu().double().numpy().reshape(KV, 2, D), k[:, :n]) * D ** -0.5
                    w = np.exp(s - s.max(-1, keepdims=True))
                    want = np.einsum("hgn,hnd->hgd", w / w.sum(-1, keepdims=True), v[:, :n]).reshape(H, D)
                    # weights and the output rounded to bf16: half a step (2^-9 relative) each, on values of some units
                    assert np.abs(out[3 * b + i] - want).max() <= 2.0 ** -8 * 4
            continue
        for x in (k_new, v_new, q_new):
            x.copy_(torch.randn(x.shape, generator=g))
        sent = [x.cpu().clone() for x in (k_new, v_new)]
        torch.cuda.synchronize()
        step.replay()
        torch.cuda.synchronize()
        for b, n in enumerate(ctx.tolist()):
            k, v = held(K, b, False, n), held(V, b, True, n)
            assert np.array_equal(k[:, n - 1], from_fp4(*to_fp4(turned(sent[0][b].double().numpy(), angles, n - 1, True)[0])))
            assert np.array_equal(v[:, n - 1], from_fp4(*to_fp4(sent[1][b].double().numpy())))
            seen = [p for p in range(n) if p >= n - window or p < sinks]
            s = np.einsum("hgd,hnd->hgn", q_new[b].cpu().double().numpy().reshape(KV, 2, D), k[:, seen]) * D ** -0.5
            w = np.exp(s - s.max(-1, keepdims=True))
            want = np.einsum("hgn,hnd->hgd", w / w.sum(-1, keepdims=True), v[:, seen]).reshape(H, D)
            # weights as two bf16 terms (off by 2^-18), q as five digits (2^-20 of a block's largest), fp32 sums: values of some units
            assert np.abs(look.out[b].cpu().double().numpy() - want).max() <= 5e-5
    assert ctx.tolist() == [40 + 27 + 9, 1 + 27 + 9]


def test_replays_follow_lengths_and_lists(gpu_device):
    """Lengths, tables, lists and `since` are read by every replay; eager calls of the same operators, with workspaces of their own, run between them."""
    s = Setting(gpu_device)
    side = torch.cuda.Stream(device=gpu_device)
    calls = [span.prepare_paged_select(s.q, s.K, s.bounds, s.table, s.ctx, 6, since=s.since, stream=side.cuda_stream)]
    calls.append(span.prepare_paged_selected_decode_attn(s.q, s.K, s.V, s.table, s.ctx, calls[0].out, 0.125, num_splits=3, stream=side.cuda_stream))
    calls.append(span.prepare_paged_decode_attn_fp4(s.q, s.K4, s.V4, s.table, s.ctx, 0.125, num_splits=4, stream=side.cuda_stream))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for call in calls:
            call()
    for lens in ([300, 61, 60, 7, 190], [1, 320, 0, 100, 16], [17, 5, 320, 64, 161]):
        s.K.copy_(s.K.nan_to_num(nan=0.5))
        s.V.copy_(s.V.nan_to_num(nan=0.25))
        s.ctx.copy_(torch.tensor(lens, dtype=torch.int32))
        s.table.copy_(s.table.flip(0))
        torch.cuda.synchronize()
        picked = span.paged_select(s.q, s.K, s.bounds.clone(), s.table, s.ctx, 6, since=s.since)
        want = [picked, span.paged_selected_decode_attn(s.q, s.K, s.V, s.table, s.ctx, picked, 0.125, num_splits=3),
                span.paged_decode_attn_fp4(s.q, s.K4, s.V4, s.table, s.ctx, 0.125, num_splits=4)]
        torch.cuda.synchronize()
        for _ in range(3):
            graph.replay()
            torch.cuda.synchronize()
            assert same([c.out for c in calls], want)


def test_what_calls_leave_as_it_was(gpu_device):
    """Attention and reading write nothing but their outputs; a selection nothing but bounds of pages with new rows and its lists; appends nothing but their rows (tests of their own)."""
    s = Setting(gpu_device)
    kept = {n: getattr(s, n).clone() for n in ("K", "V", "K4", "V4", "q", "table", "ctx", "selected", "since")}
    s.decode()
    s.decode_spans()
    s.chosen()
    s.read()
    s.bounds.fill_(7.0)
    s.since.copy_(s.ctx - 1)
    since = s.since.clone()
    s.select()
    assert same([getattr(s, n) for n in kept if n != "since"], [kept[n] for n in kept if n != "since"]) and torch.equal(s.since, since)
    touched = {int(s.table[b, (n - 1) // P]) for b, n in enumerate(LENS)}
    rest = [i for i in range(s.bounds.shape[0]) if i not in touched]
    assert bool((s.bounds[rest] == 7.0).all()) and not bool((s.bounds[sorted(touched)] == 7.0).all())
