"""Span lists over pages that span_validate refuses: the result is unspecified, yet the call ends, reads and writes nothing outside its arrays and the pool, and the
other sequences of the batch get theirs."""
import numpy as np
import pytest
import torch

import paper_2404_09336_amd as span
from paged_reference import attend

pytestmark = pytest.mark.gpu

CAP = 1 << 22
TOP = 2 ** 31 - 1
LISTS = {
    # 100 positions and 2^32: in 32 bits 100, whose rows a walk over the chunks of 64 intervals steps over
    "wraps": [(0, 100)] + [(0, 0)] * 703 + [(0, CAP)] * 1024,
    "wraps to a negative count": [(0, CAP)] * 600,
    "wraps to a few": [(0, CAP)] * 1024 + [(7, 500)],
    "outside": [(-50, 20), (CAP - 10, CAP + 300), (TOP - 3, TOP), (-TOP - 1, -TOP + 40), (2 * CAP, 2 * CAP + 70)],
    "outside, many": [(k * 70000 - CAP // 2, k * 70000 - CAP // 2 + 9) for k in range(130)],
    "reversed": [(90, 10), (300, 200), (5, 5), (TOP, -TOP - 1)],
    "overlapping": [(0, 400), (100, 500), (399, 400)] * 30,
}


@pytest.mark.parametrize("name", LISTS)
@pytest.mark.parametrize("dtype,head_dim", [("f16", 64), ("f32", 128)])
@pytest.mark.parametrize("num_splits", [0, 1])
@pytest.mark.parametrize("with_weights", [False, True])
def test_lists_that_are_refused(name, dtype, head_dim, num_splits, with_weights, gpu_device):
    dt = {"f16": torch.float16, "f32": torch.float32}[dtype]
    g = torch.Generator().manual_seed(1)
    P, KV, H = 1024, 1, 2
    K, V = (torch.randn((4, KV, P, head_dim), generator=g).to(dt) for _ in range(2))
    table = torch.randint(0, 4, (3, CAP // P), generator=g).to(torch.int32)
    q = torch.randn((3, H, head_dim), generator=g).to(dt)
    good = [(3, 40), (1500, 1900)]
    lists = [good, LISTS[name], [(0, 77)]]
    off = np.cumsum([0] + [len(x) for x in lists]).astype(np.int32)
    st, en = (np.array([iv[k] for x in lists for iv in x], np.int32) for k in (0, 1))
    dev = [torch.from_numpy(a).to(gpu_device) for a in (off, st, en)]
    room = torch.full((5, KV, CAP), 0.75, device=gpu_device)  # the call's weights lie in the middle
    Kd, Vd = K.to(gpu_device), V.to(gpu_device)
    got = span.paged_span_decode_attn(q.to(gpu_device), Kd, Vd, table.to(gpu_device), *dev, head_dim ** -0.5, num_splits=num_splits,
                                      weights=room[1:4] if with_weights else None).cpu().double()
    torch.cuda.synchronize()
    assert torch.equal(Kd.cpu(), K) and torch.equal(Vd.cpu(), V)
    assert (room[0] == 0.75).all() and (room[4] == 0.75).all()

    class Of:
        heads, kv_heads = H, KV
        rows = staticmethod(lambda pool, b, p: pool[table[b, torch.as_tensor(p) // P].long(), :, torch.as_tensor(p) % P].transpose(0, 1).double())
    Of.head_dim = head_dim
    for b in (0, 2):
        p = [x for s, e in lists[b] for x in range(s, e)]
        out, w = attend(Of, K, V, b, q[b], p, head_dim ** -0.5)
        assert float((got[b] - out).abs().max()) <= 1e-5  # as for all one-token calls
        want = torch.full((KV, CAP), 0.75, dtype=torch.float64)
        if with_weights:
            want[:, p] += w
        assert float((room[1 + b].cpu().double() - want).abs().max()) <= 2e-5  # two heads' weights
