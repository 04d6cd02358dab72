"""Prompt attention with large scores that lie close to one another: the contenders for a token's weight are spread over tiles and over workgroups that share
them, so that the largest score of the ones before is overtaken again and again."""
import numpy as np
import pytest
import torch

from test_gpu_paged_prompt import STEP, Prompt
import paper_2404_09336_amd as span

pytestmark = pytest.mark.gpu

# 4194304 / log2(e) = 2907269.7: the scores of CROSSING pass 2^22 of the kernel's units among the tiles, those below it lie wholly under or over it.
CROSSING = 2907264


@pytest.mark.parametrize("dtype,head_dim", [("f32", 64), ("f32", 128), ("f16", 128), ("bf16", 64)])
@pytest.mark.parametrize("base", [0, 1 << 10, 1 << 13, 1 << 17, 1 << 21, CROSSING, 1 << 22])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("few", [False, True])
def test_large_scores_close_to_one_another(dtype, head_dim, base, sign, few, gpu_device):
    """Scores sign * base + half of (the position's number of 32 + its lowest bit), exact in fp32: of at most 24 bits, as are all partial sums.  Few: one
    sequence, whose tiles are shared; else 256 workgroups, each with its tile."""
    heads, lens = (2, [330]) if few else (32, [300, 301, 290, 333, 310, 300, 299, 320])
    p = Prompt(lens, [20] * len(lens), heads, heads, head_dim, 16, dtype, gpu_device, seed=base % 89 + few)
    p.q.zero_()
    p.q[..., 0], p.q[..., 1], p.q[..., 2], p.q[..., 3] = 256, 256, 1, 1
    for b, n in enumerate(lens):
        for i in range(-(-n // 16)):
            rows = min(16, n - 16 * i)
            at = torch.arange(16 * i, 16 * i + rows)
            k = torch.zeros((rows, head_dim))
            k[:, 0], k[:, 1], k[:, 2] = sign * (base >> 16) * 256, sign * (base >> 8 & 255), sign * (base & 255)  # digits of the base, exact in every type
            k[:, 3] = (at // 32 + at % 2) / 2
            p.K[p.table[b, i], :, :rows] = k.to(p.K.dtype)
            v = torch.rand((heads, rows, head_dim), generator=p.generator) * 2 - 1
            p.V[p.table[b, i], :, :rows] = v.to(p.V.dtype)
    q, K, V, table, ctx, off = p.to("q", "K", "V", "table", "ctx", "off")
    got = span.paged_prompt_attn(q, K, V, table, ctx, off, 1.0).cpu().double()
    # Scores are exact.  A weight's exponent is off by less than 2^-20 (two roundings of at most half a step of values below 16), so is each rescaling of the ones
    # before, whose share falls by e^-0.5 a tile: with exp2's own steps below 1e-5 in all against values of at most 1.  16 bits: a rounding of each weight, which the sum of
    # the rounded ones passes on, and one of the output.
    for b, n in enumerate(lens):
        first = int(p.off[b])
        k, v = p.rows(p.K, b, range(n)), p.rows(p.V, b, range(n))
        sees = torch.arange(n) <= torch.arange(n - 20, n)[:, None]
        score = torch.matmul(p.q[first:first + 20].double().transpose(0, 1), k.transpose(1, 2).contiguous())
        w = torch.softmax(torch.where(sees, score, torch.tensor(-np.inf, dtype=torch.float64)), -1)
        want, size = torch.matmul(w, v).transpose(0, 1), torch.matmul(w, v.abs()).transpose(0, 1)
        allowed = 1e-5 + STEP[dtype] * (1 + 2 * STEP[dtype]) * (size + 2 * want.abs())
        over = (got[first:first + 20] - want).abs() - allowed
        assert float(over.max()) <= 0, (b, float((got[first:first + 20] - want).abs().max()))
