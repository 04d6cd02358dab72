"""Appends and reads of more waves than a launch numbers are refused, from the number of tokens on that the header gives."""
import ctypes

import pytest

from paper_2404_09336_amd import paged
from test_paged_abi import FAR, call, desc

WAVES = 1 << 26


def least_refused(kib, rows, head_dim, size, group):
    """Tokens from which a call is refused: waves of so many KiB of `rows` rows a token, tokens rounded up to `group`."""
    each = -(-rows * head_dim * size // (kib << 10))
    return (WAVES - 1) // each // group * group + 1


@pytest.mark.parametrize("heads,kv_heads,head_dim,dtype,size", [(32, 8, 128, 1, 2), (32, 32, 128, 2, 2), (1, 1, 64, 0, 4), (65535, 65535, 128, 0, 4), (96, 6, 64, 0, 4)])
@pytest.mark.parametrize("more", [0, 1, 7, 1000])
def test_the_first_that_is_refused(heads, kv_heads, head_dim, dtype, size, more):
    turn = ctypes.byref(paged._Rotation(FAR, 100, 64, 0))
    plain, fp4, read = (least_refused(12, 2 * kv_heads + heads, head_dim, size, 4), least_refused(4, 2 * kv_heads + heads, head_dim, size, 8), least_refused(4, 2 * kv_heads, head_dim, size, 8))
    tokens = lambda n: desc(batch=1, heads=heads, kv_heads=kv_heads, head_dim=head_dim, dtype_code=dtype, num_tokens=n + more)  # noqa: E731
    assert min(plain, fp4, read) >= 512
    assert call("paged_append_rotary", tokens(plain), turn, *[FAR] * 11) == -2
    assert call("paged_append_fp4", tokens(fp4), turn, *[FAR] * 10) == -2
    assert call("paged_read_fp4", tokens(read), *[FAR] * 7) == -2


def test_figures_of_the_header():
    assert least_refused(12, 2 * 8 + 32, 128, 2, 4) > (1 << 26) - 4 and 22 < least_refused(4, 2 * 8 + 32, 128, 2, 8) / 1e6 < 23


def test_few_tokens_of_very_many_heads():
    """2 KiB a wave below 512 tokens: 18 * 65535 rows of 512 bytes are 294908 waves a token, of 228 (rounded up to four) 2^26."""
    for tokens in (225, 228, 511):
        d = desc(batch=1, heads=16 * 65535, kv_heads=65535, head_dim=128, dtype_code=0, num_tokens=tokens)
        turn = ctypes.byref(paged._Rotation(FAR, 100, 64, 0))
        assert call("paged_append_fp4", d, None, *[FAR] * 10) == -2 and call("paged_append_rotary", d, turn, *[FAR] * 11) == -2
