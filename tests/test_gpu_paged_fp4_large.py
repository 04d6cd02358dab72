"""One-token attention over pages of 4-bit values as large as they get: outputs are means of what the pages hold and stay finite, however the weights are held on the way."""
import numpy as np
import pytest
import torch

import paper_2404_09336_amd as span
from paged_more_reference import place, pool_fp4, read_fp4
from test_gpu_paged_fp4_attn import Fp4Pages, check

pytestmark = pytest.mark.gpu

SHAPES = [(32, 8, 128, "bf16"), (4, 4, 64, "f32"), (14, 2, 64, "f16"), (16, 1, 128, "f32"), (8, 1, 128, "bf16")]


def scaled_values(pages, exponent, rows=slice(None), blocks=slice(None)):
    """V's blocks of those rows of a page with exponents that are so much larger, 125 at most (what is NaN stays)."""
    pool = pages.pools[1]
    N, KV, P, W = pool.shape
    D = W // 17 * 32
    flat = pool.view(N, KV, -1)
    for row in range(P)[rows]:
        at = torch.from_numpy(place(P, D, row, True)[1][blocks]).to(pool.device)
        byte = flat[..., at].int()
        flat[..., at] = torch.where(byte == 255, byte, (byte + exponent).clamp(1, 252)).to(torch.uint8)
    pages.values[1] = read_fp4(pool.cpu().numpy(), True)


def attended(pages, device, scale, **kw):
    out = span.paged_decode_attn_fp4(pages.q.to(device), *pages.cache(), pages.ctx.to(device), scale, **kw)
    assert out.isfinite().all()
    for b, n in enumerate(pages.lens):
        check(pages, out, b, range(n), scale)


@pytest.mark.parametrize("exponent", [64, 70, 100, 110, 118, 130])
@pytest.mark.parametrize("heads,kv_heads,head_dim,dtype", SHAPES)
def test_every_value_is_large(exponent, heads, kv_heads, head_dim, dtype, gpu_device):
    """Weights that are alike and up to tens of thousands of times their reference; one wave, all of them, several slices."""
    lens = [1, 20, 300, 3000, 5000]
    pages = Fp4Pages(lens, heads, kv_heads, head_dim, 16, dtype, gpu_device, seed=exponent)
    scaled_values(pages, exponent)
    for scale in (0.01, head_dim ** -0.5, 0.6):
        attended(pages, gpu_device, scale)
        attended(pages, gpu_device, scale, num_splits=3)


@pytest.mark.parametrize("heads,kv_heads,head_dim,dtype", SHAPES)
@pytest.mark.parametrize("rows,blocks", [(slice(5, 6), slice(None)), (slice(None), slice(1, 2)), (slice(3, 16, 7), slice(0, 1))])
def test_some_values_are_large(heads, kv_heads, head_dim, dtype, rows, blocks, gpu_device):
    """One row of a unit, one block of every row: its channels are its sums', and the others' as exact as ever."""
    pages = Fp4Pages([40, 1, 2500], heads, kv_heads, head_dim, 16, dtype, gpu_device, seed=5)
    scaled_values(pages, 120, rows, blocks)
    attended(pages, gpu_device, head_dim ** -0.5)


@pytest.mark.parametrize("where", [0, 31, 32, 200, 999])
@pytest.mark.parametrize("heads,kv_heads,head_dim,dtype", SHAPES)
def test_one_large_row(where, heads, kv_heads, head_dim, dtype, gpu_device):
    """Its weight is whatever it is: of nothing to nearly all."""
    for size in (-30.0, 0.0, 30.0):
        pages = Fp4Pages([1000], heads, kv_heads, head_dim, 1024, dtype, gpu_device, seed=where)
        pages.q[:] = 1
        key = np.zeros((1, kv_heads, 1024, head_dim))
        key[:, :, where] = size / head_dim
        held = read_fp4(pool_fp4(key, False), False)
        page = int(pages.table[0, 0])
        pages.pools[0][page] = torch.from_numpy(pool_fp4(key, False)[0]).to(gpu_device)
        pages.values[0][page] = held[0]
        scaled_values(pages, 122, slice(where, where + 1))
        attended(pages, gpu_device, 1.0)


@pytest.mark.parametrize("heads,kv_heads,head_dim,dtype", SHAPES)
def test_small_values_stay(heads, kv_heads, head_dim, dtype, gpu_device):
    """Values of 2^-90 and less without a large one beside them."""
    pages = Fp4Pages([300, 2000], heads, kv_heads, head_dim, 16, dtype, gpu_device, seed=2)
    scaled_values(pages, -90)
    out = span.paged_decode_attn_fp4(pages.q.to(gpu_device), *pages.cache(), pages.ctx.to(gpu_device), 0.1)
    for b, n in enumerate(pages.lens):
        want, bound = pages.attend(b, range(n), 0.1)
        bound -= 1e-30  # (the reference's own allowance, as large as these)
        assert np.all(np.abs(out[b].cpu().double().numpy() - want) <= bound) and np.abs(want).min() > 0


@pytest.mark.parametrize("head_dim", [64, 128])
def test_nan_beside_large_values(head_dim, gpu_device):
    """Only its own channels become NaN; in a row that nobody attends it does nothing."""
    pages = Fp4Pages([100, 100], 8, 2, head_dim, 16, "bf16", gpu_device)
    scaled_values(pages, 120)
    pool = pages.pools[1]
    pool.view(pool.shape[0], 2, -1)[int(pages.table[0, 2]), 1, int(place(16, head_dim, 37 % 16, True)[1][1])] = 255
    args = (pages.q.to(gpu_device), *pages.cache(), pages.ctx.to(gpu_device), 0.125)
    out = span.paged_decode_attn_fp4(*args)
    assert out[0, :4].isfinite().all() and out[1].isfinite().all() and out[0, 4:, 32:64].isnan().all() and out[0, 4:, :32].isfinite().all()
    assert span.paged_decode_attn_fp4(*args, window=62, sinks=37).isfinite().all()
