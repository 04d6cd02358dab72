"""One-token attention over pages of 4-bit values: how the states of waves, of slices and of a weight's terms become one, for every number of query heads that share a KV head."""
import numpy as np
import pytest
import torch

import paper_2404_09336_amd as span
from paged_more_reference import pool_fp4, read_fp4
from test_gpu_paged_fp4_attn import Fp4Pages, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 6, 7, 8, 9, 12, 13, 16])
@pytest.mark.parametrize("head_dim,dtype", [(64, "f16"), (128, "bf16"), (128, "f32")])
def test_several_slices(group, head_dim, dtype, gpu_device):
    """Fewer slices than a joining team has places, as many, and several rounds of them; long, short and empty sequences."""
    lens = [9000, 0, 130, 4111, 1, 700]
    pages = Fp4Pages(lens, 2 * group, 2, head_dim, 64, dtype, gpu_device, seed=group)
    for splits in (0, 2, 3, 5, 8, 9, 17, 40):
        out = torch.full((len(lens), 2 * group, head_dim), float("nan"), device=gpu_device)
        span.paged_decode_attn_fp4(pages.q.to(gpu_device), *pages.cache(), pages.ctx.to(gpu_device), 0.2, out, num_splits=splits)
        for b, n in enumerate(lens):
            check(pages, out, b, range(n), 0.2)


@pytest.mark.parametrize("group", [1, 4, 6, 8, 11, 16])
def test_several_slices_of_spans(group, gpu_device):
    """Slices from the host's counts, of unlike number, and given ones."""
    lists = [[(0, 48), (700, 2900), (3000, 5003)], [(10, 20)], [], [(5, 1500), (1600, 3333)]]
    pages = Fp4Pages([5003] * 4, group, 1, 128, 32, "bf16", gpu_device, seed=group)
    off = np.cumsum([0] + [len(x) for x in lists]).astype(np.int32)
    st, en = (np.asarray([iv[i] for x in lists for iv in x], np.int32) for i in (0, 1))
    tokens = np.asarray([sum(e - s for s, e in x) for x in lists], np.int64)
    args = [torch.from_numpy(x).to(gpu_device) for x in (off, st, en)]
    for kw in ({}, {"tokens_per_seq": tokens}, {"num_splits": 2}, {"num_splits": 11}):
        out = span.paged_span_decode_attn_fp4(pages.q.to(gpu_device), *pages.cache(), *args, 0.1, **kw)
        for b, x in enumerate(lists):
            check(pages, out, b, [p for s, e in x for p in range(s, e)], 0.1)


@pytest.mark.parametrize("group", [1, 3, 4, 5, 7, 8, 9, 14, 16])
@pytest.mark.parametrize("head_dim,dtype", [(64, "f32"), (64, "bf16"), (128, "f32"), (128, "f16")])
@pytest.mark.parametrize("order", [0, 1])
def test_weights_meet_v_whole(group, head_dim, dtype, order, gpu_device):
    """Row p of V is 1 in one channel of its own and 0 elsewhere: outputs are the weights themselves, so that a lost or misplaced term of one shows."""
    n, KV = head_dim, 2
    rng = np.random.default_rng(100 * group + head_dim + order)
    pages = Fp4Pages([n], KV * group, KV, head_dim, n, dtype, gpu_device, seed=group)
    q = rng.integers(1, 16, (1, KV * group, head_dim)) * rng.choice([-1, 1], (1, KV * group, head_dim)) / 8  # (four bits: exact in every type)
    pages.q = torch.from_numpy(q).to(pages.q.dtype)
    value = np.zeros((1, KV, n, head_dim))
    value[0, :, np.arange(n), np.arange(n) if order == 0 else rng.permutation(n)] = 1
    page = int(pages.table[0, 0])
    pool = pool_fp4(value, True)
    assert np.array_equal(read_fp4(pool, True), value)
    pages.pools[1][page] = torch.from_numpy(pool[0]).to(gpu_device)
    scale = 2.0 ** -12
    out = span.paged_decode_attn_fp4(pages.q.to(gpu_device), *pages.cache(), pages.ctx.to(gpu_device), scale)[0].cpu().double().numpy()
    k = pages.values[0][page].astype(np.float64)                                             # [KV, n, D]
    q = q.reshape(KV, group, head_dim)
    s = scale * q @ k.transpose(0, 2, 1)
    w = np.exp(s - s.max(-1, keepdims=True))
    want = (w / w.sum(-1, keepdims=True) @ value[0]).reshape(KV * group, head_dim)
    # Scores as for the other tests: a channel of q is off by 2^-20 of its block's largest (up to 15/8), a score's roundings by 2^-20 of its products; twice the largest difference of scores.
    size = scale * (15 / 8 + np.abs(q)) @ np.abs(k).transpose(0, 2, 1) * 2.0 ** -20
    # In units of 2^-24, above and below the division, each relative to a weight of about 1: the argument's rounding (1 each), exp2 (2 each), the factor that joins the waves (2), its product and
    # sum (2), each twice; the sum's own chain: 4 of a step of 32 positions, of which a wave has one, 2 over the lanes, 4 over the waves; the division.
    # A weight's 24 bits go in whole, and all other products of its channel are zero.
    off = np.expm1(2 * size.max()) + (2 * (1 + 2 + 2 + 2) + 10 + 1) * 2.0 ** -24
    assert np.all(np.abs(out - want) <= off * want)
    # (that notices two terms in place of three: the nearest numbers of 16 bits are further off, here and there)
    w32 = w.astype(np.float32)
    mantissa, exponent = np.frexp(w32)
    two = np.ldexp(np.round(mantissa * 65536) / 65536, exponent)
    assert np.any(np.abs(two / w32 - 1) > 2 * off)
