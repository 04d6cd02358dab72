"""Calls on a cache in pages as programs make them: refusals of the binding, streams, calls side by side, a workspace that serves several operators."""
import pytest
import torch

import paper_2404_09336_amd as span
from paged_reference import Pages

pytestmark = pytest.mark.gpu

B, H, KV, D, P, BUDGET = 5, 8, 2, 64, 16, 60
LENS = [300, 61, 60, 7, 190]


def same(a, b):
    return all(torch.equal(x.cpu().contiguous().view(torch.uint8), y.cpu().contiguous().view(torch.uint8)) for x, y in zip(a, b))


class Setting:
    def __init__(self, device, seed=0):
        pages = Pages(LENS, H, KV, D, P, "f16", device, seed=seed, table_pages=20)
        self.K, self.V, self.table, self.ctx = pages.to("K", "V", "table", "ctx")
        self.cache = (self.K, self.V, self.table)
        g = pages.generator
        slots = (B, KV, pages.capacity)
        self.q = pages.q.to(device)
        self.weights = torch.rand(slots, generator=g).to(device)
        self.positions = torch.arange(pages.capacity, dtype=torch.int32).expand(slots).contiguous().to(device)
        self.new = [torch.randn((B, KV, D), generator=g).half().to(device) for _ in range(2)]
        self.prompt = torch.randn((B * 3, H, D), generator=g).half().to(device)
        self.offsets = torch.arange(0, 3 * B + 1, 3, dtype=torch.int32, device=device)
        self.spans = [torch.tensor(x, dtype=torch.int32, device=device) for x in
                      ([0, 2, 3, 4, 5, 6], [0, 250, 10, 0, 3, 100], [20, 300, 61, 60, 7, 130])]

    def attend(self, **kw):
        return span.paged_decode_attn(self.q, *self.cache, self.ctx, 0.125, **kw)

    def attend_spans(self, **kw):
        return span.paged_span_decode_attn(self.q, *self.cache, *self.spans, 0.125, **kw)

    def attend_prompt(self, **kw):
        return span.paged_prompt_attn(self.prompt, *self.cache, self.ctx, self.offsets, 0.125, **kw)

    def evict(self, **kw):
        return span.paged_evict(*self.cache, self.ctx, self.weights, BUDGET, sinks=2, recent=9, positions=self.positions, **kw)

    def append(self, **kw):
        return span.paged_append(*self.new, *self.cache, self.ctx, **kw)


def misaligned(t):
    """The same values one element (of less than 16 bytes) off."""
    store = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
    store[1:] = t.reshape(-1)
    return store[1:].view(t.shape)


@pytest.mark.parametrize("what", ["K", "V", "table", "ctx", "q", "weights", "positions", "new", "prompt", "offsets", "spans"])
def test_refused_tensors(what, gpu_device):
    """Another type, another shape, not contiguous, not aligned, not on the GPU: each tensor, in a call that takes it, before anything is launched."""
    s = Setting(gpu_device)
    calls = {"K": s.attend, "V": s.attend, "table": s.append, "ctx": s.evict, "q": s.attend, "weights": s.evict, "positions": s.evict, "new": s.append,
             "prompt": s.attend_prompt, "offsets": s.attend_prompt, "spans": s.attend_spans}
    call = calls[what]
    call()
    before = {n: getattr(s, n).clone() for n in ("K", "V", "weights", "positions")}
    good = getattr(s, what)
    if what in ("new", "spans"):
        variants = lambda f: [good[0], f(good[1]), *good[2:]]  # noqa: E731
        one = good[1]
    else:
        variants = lambda f: f(good)  # noqa: E731
        one = good
    other_shape = lambda t: torch.cat((t, t), dim=0 if what == "table" else t.dim() - 1)[..., :-1].contiguous()  # noqa: E731
    doubled = lambda t: torch.stack((t, t), dim=-1)[..., 0]  # noqa: E731
    bad = [lambda t: t.double() if t.is_floating_point() else t.long(), other_shape, doubled, misaligned, lambda t: t.cpu()]
    assert not doubled(one).is_contiguous() and misaligned(one).data_ptr() % 16 != 0
    for f in bad:
        setattr(s, what, variants(f))
        s.cache = (s.K, s.V, s.table)
        with pytest.raises((ValueError, span.SpanAttnError)):
            call()
    setattr(s, what, good)
    s.cache = (s.K, s.V, s.table)
    assert same([getattr(s, n) for n in before], before.values())


def test_refused_arguments(gpu_device):
    s = Setting(gpu_device)
    for call in (lambda: s.evict(positions_out=s.positions[:, :1].contiguous()), lambda: s.evict(new_lens=s.ctx.long()),
                 lambda: span.paged_evict(*s.cache, s.ctx, s.weights, 0), lambda: span.paged_evict(*s.cache, s.ctx, s.weights, 10, sinks=5, recent=6),
                 lambda: span.paged_evict(*s.cache, s.ctx, s.weights, 10, positions_out=s.positions), lambda: s.attend(window=-1),
                 lambda: s.attend(workspace=torch.zeros(64, dtype=torch.uint8, device=gpu_device)),
                 lambda: s.attend(out=torch.empty((B, H, D), dtype=torch.float16, device=gpu_device)), lambda: s.attend(weights=s.weights[:, :1].contiguous()),
                 lambda: span.paged_append(s.new[0], s.new[1], *s.cache, s.ctx, seen=s.ctx[:2].contiguous()),
                 lambda: span.paged_decode_attn(s.q[:, :7].contiguous(), *s.cache, s.ctx, 0.125),
                 lambda: span.paged_decode_attn(s.q[0], *s.cache, s.ctx, 0.125)):
        with pytest.raises((ValueError, span.SpanAttnError)):
            call()


def results(s, **kw):
    """All operators in the order a step runs them; the caches are the setting's own."""
    s.append(positions=s.positions, **kw)
    out = [s.attend(weights=s.weights, **kw), s.attend_spans(**kw), s.attend_prompt(**kw)]
    return [*out, *s.evict(**kw), s.K, s.V, s.weights, s.positions]


def test_another_stream_while_the_current_one_is_busy(gpu_device):
    """New outputs and workspaces belong to the call's stream: what the current stream still has to do neither comes between nor overwrites them."""
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


def test_one_workspace_for_all_one_token_calls_and_evictions(gpu_device):
    """Every call leaves the counters zero: calls that follow one another share a workspace, initialised once."""
    want = results(Setting(gpu_device))
    s = Setting(gpu_device)
    shared = torch.empty(1 << 22, dtype=torch.uint8, device=gpu_device)
    call = span.prepare_paged_evict(*s.cache, s.ctx, s.weights, BUDGET, workspace=shared)  # (for its descriptor)
    span.paged_workspace_init(call.desc)
    for _ in range(3):
        s = Setting(gpu_device)
        s.append(positions=s.positions)
        out = [s.attend(weights=s.weights, workspace=shared), s.attend_spans(workspace=shared), s.attend_prompt()]
        assert same([*out, *s.evict(workspace=shared), s.K, s.V, s.weights, s.positions], want)
        # in place, which takes tickets
        t = Setting(gpu_device)
        t.append(positions=t.positions)
        t.attend(weights=t.weights, workspace=shared)
        t.evict(workspace=shared, weights_out=t.weights, positions_out=t.positions, new_lens=t.ctx)
        assert torch.equal(t.ctx.cpu(), want[5].cpu()) and same([t.K, t.V], [s.K, s.V])
