"""Rotated appends that turn all channels of a row of 128, or nearly all: the other channel of a pair is up to 16 lanes away, and no lane of a row stays as it is."""
import numpy as np
import pytest
import torch

import paper_2404_09336_amd as span
from paged_more_reference import place, rotation_table, to_fp4, turned
from paged_reference import DTYPES
from test_gpu_paged_turned import MANY, MANY_LENS, Rows, check_fp4, check_rotary

pytestmark = pytest.mark.gpu

CHANNELS = [(128, False), (128, True), (112, False), (112, True), (96, False)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads,kv_heads", [(2, 1), (9, 3), (40, 40)])
@pytest.mark.parametrize("channels,paired", CHANNELS)
@pytest.mark.parametrize("new", ["one", "some", "many"])
def test_rotary(dtype, heads, kv_heads, channels, paired, new, gpu_device):
    if new == "many":
        heads, kv_heads = min(heads, 11), min(kv_heads, 11)
        r = Rows(MANY, heads, kv_heads, 128, dtype, gpu_device, seed=channels, ahead=30, lens=MANY_LENS)
    else:
        r = Rows(new, heads, kv_heads, 128, dtype, gpu_device, seed=channels, ahead=30)
    check_rotary(r, dtype, kv_heads, channels, paired, gpu_device)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads,kv_heads", [(2, 1), (9, 3), (18, 18)])
@pytest.mark.parametrize("channels,paired", CHANNELS)
@pytest.mark.parametrize("new", ["one", "some", "many"])
def test_fp4(dtype, heads, kv_heads, channels, paired, new, gpu_device):
    if new == "many":
        r = Rows(MANY, heads, kv_heads, 128, dtype, gpu_device, seed=channels + 1, ahead=30, lens=MANY_LENS)
    else:
        r = Rows(new, heads, kv_heads, 128, dtype, gpu_device, seed=channels + 1, ahead=30)
    check_fp4(r, dtype, kv_heads, 128, channels, paired, gpu_device)


@pytest.mark.parametrize("paired", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [40, 640])
def test_values_next_to_borders(dtype, paired, n, gpu_device):
    """Values that are a few units of fp32 and less from a border, or on it, in every block of a row; of a step's tokens and of a prompt's."""
    D, KV = 128, 2
    g = torch.Generator().manual_seed(n)
    x = torch.randn((n, KV, D), generator=g) * 2.0 ** torch.randint(-6, 7, (n, KV, 1), generator=g)
    angles = rotation_table(n, D)
    one = list(range(0, D, 2)) if paired else list(range(64))
    two = list(range(1, D, 2)) if paired else list(range(64, D))
    for t in range(0, n, 2):  # angle 0 and almost: x cos - x' sin = border + j tiny
        angles[t, :64], angles[t, 64:] = 1.0, 2.0 ** -18
        for i in range(64):
            x[t, 0, one[i]] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0][(t // 2 + i) % 8] * (1 if i % 3 else -1)
            x[t, 0, two[i]] = float(torch.randint(-3, 4, (1,), generator=g)) * 2.0 ** -(6 + t % 8)
    x = x.to(DTYPES[dtype])
    K, V = (span.fp4_pages(40, KV, 16, D, gpu_device) for _ in range(2))
    table = torch.arange(40, dtype=torch.int32, device=gpu_device)[None].contiguous()
    ctx, off = torch.tensor([n], dtype=torch.int32, device=gpu_device), torch.tensor([0, n], dtype=torch.int32, device=gpu_device)
    xg = x.to(gpu_device)
    span.paged_append_fp4(xg, xg, K, V, table, ctx, off, rotation=angles.to(gpu_device), paired=paired)
    flat = K.cpu().reshape(40, KV, -1).numpy()
    for t in range(n):
        code, byte = to_fp4(turned(x[t].double().numpy(), angles, t, paired)[0])
        codes, exps = place(16, D, t % 16, False)
        for h in range(KV):
            assert np.array_equal(flat[t // 16, h][exps], byte[h]), (t, h)
            assert np.array_equal(flat[t // 16, h][codes], code[h][0::2] | (code[h][1::2] << 4)), (t, h)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_positions_without_angles(dtype, gpu_device):
    """All of a row becomes NaN, K's and q's; V and everybody else stay."""
    r = Rows("one", 4, 2, 128, dtype, gpu_device)
    angles = rotation_table(64, 128)
    K, V, table, ctx = r.pages.to("K", "V", "table", "ctx")
    k, v, q = r.on(gpu_device, "k", "v", "q")
    seen = torch.tensor([64, 65, 0, -5, 1, 2, 1 << 30, 4], dtype=torch.int32)  # positions 63, 64, -1, -6, 0, 1, far, 3
    out = span.paged_append_rotary(k, v, K, V, table, ctx, angles.to(gpu_device), q=q, seen=seen.to(gpu_device))[2].cpu()
    assert out[[1, 2, 3, 6]].isnan().all() and not out[[0, 4, 5, 7]].isnan().any()
    for b in (1, 2, 3):
        page, at = r.slot(b, r.pages.ctx[b].item() - 1)
        assert K[page, :, at].isnan().all() and torch.equal(V[page, :, at].cpu(), r.v[b])
