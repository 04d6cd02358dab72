"""Plain 64-bit forms of the operators on a cache in pages, and random caches for their tests."""
import numpy as np
import torch

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


class Pages:
    """Random pools whose pages the sequences hold in random order; what no sequence holds is NaN, and so are the rows past a sequence's length."""

    def __init__(self, lens, heads, kv_heads, head_dim, page, dtype, device, seed=0, table_pages=None, spare=3):
        self.lens, self.heads, self.kv_heads, self.head_dim, self.page = list(lens), heads, kv_heads, head_dim, page
        g = torch.Generator().manual_seed(seed)
        B = len(self.lens)
        self.table_pages = table_pages or max(1, max(-(-n // page) for n in self.lens))
        pages = B * self.table_pages + spare
        self.table = torch.randperm(pages, generator=g)[:B * self.table_pages].reshape(B, self.table_pages).to(torch.int32)
        shape = (pages, kv_heads, page, head_dim)
        dt = DTYPES[dtype]
        self.K, self.V = (torch.full(shape, float("nan"), dtype=dt) for _ in range(2))
        for b, n in enumerate(self.lens):
            for i in range(-(-n // page)):
                rows = min(page, n - i * page)
                for pool in (self.K, self.V):
                    pool[self.table[b, i], :, :rows] = torch.randn((kv_heads, rows, head_dim), generator=g).to(dt)
        self.q = torch.randn((B, heads, head_dim), generator=g).to(dt)
        self.generator, self.device = g, device
        self.ctx = torch.tensor(self.lens, dtype=torch.int32)

    def to(self, *names):
        return [getattr(self, n).to(self.device) for n in names]

    @property
    def capacity(self):
        return self.table_pages * self.page

    def rows(self, pool, b, positions):
        """[kv_heads, len(positions), head_dim] in 64 bits."""
        p = torch.as_tensor(np.asarray(positions, dtype=np.int64))
        page = self.table[b, p // self.page].long().clamp(0, pool.shape[0] - 1)  # (who names others masks what is there)
        return pool[page, :, p % self.page].transpose(0, 1).double()


def seen_positions(n, window, sinks):
    """Positions that the token at position n - 1 sees."""
    return [p for p in range(n) if window == 0 or p >= n - window or p < sinks]


def attend(pages, K, V, b, q, positions, scale):
    """(out [heads, head_dim], weights [kv_heads, positions]) of one query row, in 64 bits; zeros where there are no positions."""
    H, KV, D = pages.heads, pages.kv_heads, pages.head_dim
    if len(positions) == 0:
        return torch.zeros((H, D), dtype=torch.float64), torch.zeros((KV, 0), dtype=torch.float64)
    k, v = pages.rows(K, b, positions), pages.rows(V, b, positions)
    s = torch.matmul(q.double().reshape(KV, H // KV, D), k.transpose(1, 2).contiguous()) * scale
    w = torch.softmax(s, dim=-1)
    return torch.matmul(w, v).reshape(H, D), w.sum(1)


def evict(n, weights, positions, budget, sinks, recent):
    """Of one (sequence, KV head): slots moved to and from, in order; weights and positions are host arrays of the n slots in use."""
    if n <= budget:
        return [], []
    last = max(positions)
    order = sorted(range(n), key=lambda i: (not (positions[i] < sinks or positions[i] > last - recent),
                                            np.inf if np.isnan(weights[i]) else -weights[i], np.isnan(weights[i]), i))
    stay = set(order[:budget])
    return [i for i in range(budget) if i not in stay], sorted(i for i in stay if i >= budget)
