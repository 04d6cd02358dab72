"""Plain 64-bit forms of rotated and 4-bit appends, of 4-bit pages and of page selection."""
import numpy as np
import torch

LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
BORDERS = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5])


def rotation_table(positions, channels, base=10000.0):
    """fp32 [positions, channels]: cosines, sines."""
    angle = np.arange(positions)[:, None] * base ** (-np.arange(channels // 2) * 2.0 / channels)
    return torch.from_numpy(np.concatenate((np.cos(angle), np.sin(angle)), 1).astype(np.float32))


def turned(x, table, position, paired):
    """Row(s) x [..., head_dim] (64-bit numpy) at one position, and the sum of the products' magnitudes; NaN where the table has no such position."""
    y, size = x.copy(), np.abs(x)
    channels = table.shape[1]
    half = channels // 2
    row = np.full(channels, np.nan) if not 0 <= position < table.shape[0] else table[position].double().numpy()
    c, s = row[:half], row[half:]
    one, two = (slice(0, channels, 2), slice(1, channels, 2)) if paired else (slice(0, half), slice(half, channels))
    y[..., one], y[..., two] = x[..., one] * c - x[..., two] * s, x[..., one] * s + x[..., two] * c
    size[..., one] = np.abs(x[..., one] * c) + np.abs(x[..., two] * s)
    size[..., two] = np.abs(x[..., one] * s) + np.abs(x[..., two] * c)
    return y, size


def to_fp4(x):
    """(codes [..., D], exponent bytes [..., D / 32]) of rows of 64-bit values."""
    x = np.asarray(x, np.float64)
    block = x.reshape(*x.shape[:-1], -1, 32)
    with np.errstate(all="ignore"):
        most = np.abs(block).max(-1)
        bad = ~(most <= 7 * 2.0 ** 125)
        e = np.full(most.shape, -126)
        for k in range(-126, 126):  # the least exponent from which seven times two to it reaches
            e = np.where(most > 7 * 2.0 ** k, k + 1, e)
        y = np.abs(np.where(np.isfinite(block), block, 0)) / 2.0 ** e[..., None]
        n = np.searchsorted(BORDERS, y)                       # borders below
        n += (n < 7) & (y == BORDERS[np.minimum(n, 6)]) & (n % 2 == 1)  # on a border: the even number
        code = n + 8 * np.signbit(block)
    return code.reshape(x.shape).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def from_fp4(code, byte):
    value = LEVELS[code & 7] * np.where(code & 8, -1.0, 1.0)
    scale = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))
    return (value.reshape(*code.shape[:-1], -1, 32) * scale[..., None]).reshape(code.shape)


def place(page_rows, D, row, is_v):
    """Bytes of a (page, head) that hold a row's codes (of channels 0, 2, 4 ..) and its exponents, as span_paged.h lays them out."""
    g, r, c, w = row // 16, row % 16, np.arange(0, D, 2), D // 16
    if is_v:
        codes = g * 8 * D + r // 4 * 2 * D + c // w * 2 * w + r % 4 * (w // 2) + c % w // 2
    else:
        codes = g * 8 * D + c // 32 * 256 + r * 16 + c % 32 // 2
    return codes, page_rows * D // 2 + g * (D // 2) + np.arange(D // 32) * 16 + r


def write_fp4(flat, page_rows, D, row, is_v, code, byte):
    """A row into flat [bytes of a (page, head)]."""
    codes, exps = place(page_rows, D, row, is_v)
    flat[codes], flat[exps] = code[0::2] | (code[1::2] << 4), byte


def read_fp4(pool, is_v):
    """Values [pages, kv_heads, rows, D] in 64 bits of a pool [pages, kv_heads, rows, D / 2 + D / 32]."""
    pool = np.asarray(pool)
    N, KV, P, W = pool.shape
    D = W // 17 * 32
    flat = pool.reshape(N, KV, -1)
    out = np.zeros((N, KV, P, D))
    for row in range(P):
        codes, exps = place(P, D, row, is_v)
        two = flat[..., codes]
        code = np.stack((two & 15, two >> 4), -1).reshape(N, KV, D)
        out[:, :, row] = from_fp4(code, flat[..., exps])
    return out


def pool_fp4(values, is_v):
    """A pool [pages, kv_heads, rows, D / 2 + D / 32] that holds the nearest of `values` [pages, kv_heads, rows, D]."""
    values = np.asarray(values, np.float64)
    N, KV, P, D = values.shape
    flat = np.zeros((N, KV, P * (D // 2 + D // 32)), np.uint8)
    code, byte = to_fp4(values)
    for row in range(P):
        codes, exps = place(P, D, row, is_v)
        flat[..., codes] = code[:, :, row, 0::2] | (code[:, :, row, 1::2] << 4)
        flat[..., exps] = byte[:, :, row]
    return flat.reshape(N, KV, P, -1)


def select(q, bounds, n, pages_of, page_rows, budget, sinks, recent):
    """The list of one (sequence, KV head): q [group, D], bounds [pages of the pool, 2, D] in 64 bits, pages_of the sequence's pages."""
    count = -(-n // page_rows)
    if count <= budget:
        return list(range(count)) + [-1] * (budget - count)
    q = np.asarray(q, np.float64)
    with np.errstate(all="ignore"):
        pos, neg = np.where(np.isnan(q), q, np.maximum(q, 0)).sum(0), np.where(np.isnan(q), q, np.minimum(q, 0)).sum(0)
    rank = []
    for j in range(count):
        page = pages_of[j]
        with np.errstate(all="ignore"):
            s = np.float32((pos * bounds[page, 1] + neg * bounds[page, 0]).sum()) if 0 <= page < len(bounds) else -np.inf
        first = j * page_rows < sinks or (j + 1) * page_rows > n - max(recent, 1)
        rank.append((not first, not np.isnan(s), -s if not np.isnan(s) else 0.0, j))
    return sorted(j for *_, j in sorted(rank)[:budget])
