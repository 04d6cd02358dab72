"""More operators on a cache in pages as cases that can be timed and compared: `run` computes them from elementary torch operations (`own` false) or makes the
framework's calls (`own` true).

Keys of a case
  op        "rotate"  new rows into the pages, K and q rotated on the way                      (paged_append_rotary)
            "pack"    new rows into pages of 4-bit values, and read back as the values they stand for   (paged_append_fp4, paged_read_fp4)
            "packed"  one token per sequence over a cache of 4-bit values                      (paged_decode_attn_fp4; paged_span_decode_attn_fp4 with `spans`)
            "select"  the pages that a query scores highest by their channels' bounds          (paged_select)
            "chosen"  one token per sequence over chosen pages                                 (paged_selected_decode_attn)
  dtype     "f32" | "f16" | "bf16"
  batch, heads, kv_heads, head_dim, page
  min_len, max_len   cached positions of a sequence, the new tokens among them, drawn uniformly
  min_new, max_new   "rotate", "pack": new tokens of a sequence, drawn uniformly, at most its cached positions
  angles             "rotate", "pack": channels of a row that are rotated (0: none); `paired`: neighbours form pairs, otherwise halves do
  ahead              "rotate", "pack": how far a token's position lies past its slot (rows that were evicted)
  track              "rotate": the positions of the rows are noted
  window, sinks      "packed": a token sees the last `window` positions up to its own (0: all) and the first `sinks`
  spans              "packed": intervals of a sequence (0: no span lists)
  budget             "select", "chosen": pages of a list
  sinks, recent      "select": the first and last positions, whose pages are chosen in any case
  fresh              "select": rows of the cache's end whose bounds are not made yet (0: only the newest)
"""
import math

import numpy as np
import torch

own = False

_DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _case(name, op, dtype, batch, heads, head_dim, page, lens, **more):
    c = {"name": name, "op": op, "dtype": dtype, "batch": batch, "heads": heads[0], "kv_heads": heads[1], "head_dim": head_dim, "page": page,
         "min_len": lens[0], "max_len": lens[1]}
    return {**c, **more}


def listed():
    return [
        # what a decode step of a served batch does first, on caches that an eviction has cut
        _case("rotate-step-f16", "rotate", "f16", 64, (32, 8), 128, 16, (400, 4096), min_new=1, max_new=1, angles=128, paired=False, ahead=1000, track=True),
        # prompts of a served batch going into the cache
        _case("rotate-prompts-bf16", "rotate", "bf16", 16, (32, 8), 128, 64, (100, 4096), min_new=100, max_new=4096, angles=128, paired=False, ahead=0, track=False),
        # the same step where the cache is held in 4 bits
        _case("pack-step-bf16", "pack", "bf16", 64, (32, 8), 128, 64, (400, 4096), min_new=1, max_new=1, angles=128, paired=False, ahead=0),
        # prompts of a model that rotates half of its channels, neighbours in pairs, as many KV heads as query heads
        _case("pack-prompts-f16", "pack", "f16", 6, (32, 32), 128, 16, (333, 2500), min_new=333, max_new=2500, angles=64, paired=True, ahead=0),
        # the smallest call anybody makes: latency and launch cost only
        _case("packed-tiny-f32", "packed", "f32", 1, (4, 4), 64, 16, (256, 256), window=0, sinks=0, spans=0),
        # a served batch, four query heads per KV head, ragged
        _case("packed-batch-bf16", "packed", "bf16", 64, (32, 8), 128, 64, (512, 4096), window=0, sinks=0, spans=0),
        # self-selected spans (an instruction, a few line ranges, the recent tokens) of 16 articles, one query head per KV head
        _case("packed-span-f16", "packed", "f16", 16, (32, 32), 128, 16, (2048, 4096), window=0, sinks=0, spans=5),
        # four long documents
        _case("packed-long-bf16", "packed", "bf16", 4, (32, 8), 128, 256, (8000, 32768), window=0, sinks=0, spans=0),
        # a step of a batch of conversations: 64 of up to 512 pages of 16 are chosen
        _case("select-step-f16", "select", "f16", 64, (32, 8), 128, 16, (2000, 8192), budget=64, sinks=16, recent=64, fresh=0),
        # the first step behind long prompts, whose bounds are made on the way
        _case("select-prompt-bf16", "select", "bf16", 4, (32, 8), 128, 64, (8000, 32768), budget=32, sinks=64, recent=128, fresh=32768),
        # the attention that follows the one selection and the other
        _case("chosen-step-f16", "chosen", "f16", 64, (32, 8), 128, 16, (2000, 8192), budget=64),
        _case("chosen-long-bf16", "chosen", "bf16", 4, (32, 8), 128, 64, (8000, 32768), budget=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: batch 1 .. 64, 1 .. 32768 cached positions, caches up to 1 GiB in the storage type, prompts up to 160 MiB of new rows."""
    op = rng.choice(["rotate", "pack", "packed", "packed", "packed", "select", "select", "chosen", "chosen"])
    dtype = rng.choice(["f16", "bf16", "bf16", "f32"])
    heads = rng.choice([(32, 8), (32, 32), (16, 2), (12, 4), (14, 2), (5, 5), (8, 1), (16, 1), (6, 3)])
    head_dim = rng.choice([128, 128, 64])
    page = rng.choice([16, 32, 64, 256])
    batch, top = _log_int(rng, 1, 64), _log_int(rng, 16, 32768)
    e = 4 if dtype == "f32" else 2
    while batch * top * 2 * heads[1] * head_dim * e > 1 << 30:
        batch, top = (max(batch // 2, 1), top) if batch > 1 else (1, top // 2)
    low = max(1, int(top * rng.uniform(0.1, 1.0)))
    more = {}
    if op in ("rotate", "pack"):
        most = 1 if rng.random() < 0.5 else _log_int(rng, 1, top)
        most = max(1, min(most, (160 << 20) // (batch * (heads[0] + 2 * heads[1]) * head_dim * e)))
        more = {"min_new": max(1, int(most * rng.uniform(0.2, 1.0))), "max_new": most, "angles": rng.choice([head_dim, head_dim, head_dim // 2, 16, 48, 0 if op == "pack" else 32]),
                "paired": rng.random() < 0.3, "ahead": rng.choice([0, 0, 1000])}
        if op == "rotate":
            more["track"] = rng.random() < 0.5
    if op == "packed":
        windowed = rng.random() < 0.4
        more = {"window": _log_int(rng, 1, top) if windowed else 0, "sinks": rng.choice([0, 1, 4, 17, 64]) if windowed else 0}
        more["spans"] = rng.choice([0, 1, 7, 40]) if not windowed else 0
    if op in ("select", "chosen"):
        pages = -(-top // page)
        more = {"budget": max(4, int(pages * rng.uniform(0.05, 0.7)))}
        if op == "select":
            more.update(sinks=rng.choice([0, 1, page]), recent=rng.choice([1, page, page + 5]), fresh=rng.choice([0, 0, page, top]))
    case = _case("", op, dtype, batch, heads, head_dim, page, (low, top), **more)
    del case["name"]
    return case


def _lengths(case):
    """Cached positions and new tokens of the sequences: a case's own, which the seed puts in another order."""
    rng = np.random.default_rng([case["batch"], case["min_len"], case["max_len"]])
    lens = rng.integers(case["min_len"], case["max_len"] + 1, case["batch"]).astype(np.int64)
    lens[0] = case["max_len"]
    new = None
    if "min_new" in case:
        new = np.minimum(rng.integers(case["min_new"], case["max_new"] + 1, case["batch"]), lens)
    return lens, new


def _span_lists(case, lens, rng):
    """Sorted disjoint intervals: the beginning, some ranges in between, the recent positions."""
    off, st, en = [0], [], []
    for n in lens:
        head, tail = min(int(n), 48), max(int(n) - 64, 0)
        room = tail - head
        ranges = [(0, head)]
        if room >= 2 * case["spans"]:
            cuts = np.sort(rng.choice(room, 2 * case["spans"], replace=False)) + head
            ranges += [(int(a), int(a) + max(1, (int(b) - int(a)) // 3)) for a, b in zip(cuts[::2], cuts[1::2])]
        if tail > head:
            ranges.append((tail, int(n)))
        elif n > head:
            ranges.append((head, int(n)))
        st += [a for a, _ in ranges]
        en += [b for _, b in ranges]
        off.append(len(st))
    return [np.asarray(x, np.int32) for x in (off, st, en)]


def _nearest_fp4(x):
    """Codes (0 .. 15) and exponent bytes of rows [..., head_dim], each block of 32 channels with the least exponent from which seven times two to it reaches."""
    x = x.unflatten(-1, (-1, 32))
    most = x.abs().amax(-1, keepdim=True)
    m, k = torch.frexp(most)
    e = torch.where(most > 0, k - 3 + (m > 0.875).to(k.dtype), torch.full_like(k, -126)).clamp(min=-126)
    y = torch.ldexp(x.abs(), -e)
    code = torch.where(y < 2, torch.round(y * 2), torch.where(y < 4, torch.round(y) + 2, torch.round(y / 2) + 4)).clamp(max=7)  # (round: ties to even)
    code = code.to(torch.uint8) + 8 * torch.signbit(x).to(torch.uint8)
    return code.flatten(-2), (e[..., 0] + 127).to(torch.uint8)


def _values_of(code, byte):
    """What codes [..., head_dim] and exponent bytes [..., head_dim / 32] stand for, in 32 bits."""
    level = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=code.device)
    v = level[(code & 7).long()] * (1 - 2 * (code >> 3).float())
    return torch.ldexp(v.unflatten(-1, (-1, 32)), byte.to(torch.int32)[..., None] - 127).flatten(-2)


def _pool_fp4(code, byte, is_v):
    """Rows [pages, kv_heads, page, head_dim] as a page holds them: groups of 16 rows, of K by blocks of 32 channels and in each by rows, of V by fours of rows, in each by
    sixteenths of the channels and in those by rows; then the exponents in groups of 16 rows, by blocks and in each by rows."""
    N, KV, P, D = code.shape
    two = code[..., 0::2] | (code[..., 1::2] << 4)
    if is_v:
        rows = two.reshape(N, KV, P // 16, 4, 4, 16, D // 32).permute(0, 1, 2, 3, 5, 4, 6)
    else:
        rows = two.reshape(N, KV, P // 16, 16, D // 32, 16).permute(0, 1, 2, 4, 3, 5)
    exps = byte.reshape(N, KV, P // 16, 16, D // 32).permute(0, 1, 2, 4, 3)
    return torch.cat((rows.reshape(N, KV, -1), exps.reshape(N, KV, -1)), -1).reshape(N, KV, P, D // 2 + D // 32).contiguous()


def _unpool_fp4(pool, is_v):
    """The values of a pool's rows, [pages, kv_heads, page, head_dim] in 32 bits."""
    N, KV, P, W = pool.shape
    D = W * 32 // 17
    flat = pool.reshape(N, KV, -1)
    if is_v:
        two = flat[..., :P * D // 2].reshape(N, KV, P // 16, 4, 16, 4, D // 32).permute(0, 1, 2, 3, 5, 4, 6)
    else:
        two = flat[..., :P * D // 2].reshape(N, KV, P // 16, D // 32, 16, 16).permute(0, 1, 2, 4, 3, 5)
    two = two.reshape(N, KV, P, D // 2)
    byte = flat[..., P * D // 2:].reshape(N, KV, P // 16, D // 32, 16).permute(0, 1, 2, 4, 3).reshape(N, KV, P, D // 32)
    return _values_of(torch.stack((two & 15, two >> 4), -1).flatten(-2), byte)


def prepare(case, seed):
    torch.cuda.synchronize()
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, B, H, KV, D, P = _DTYPES[case["dtype"]], case["batch"], case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    op = case["op"]
    rng = np.random.default_rng(seed)
    order = rng.permutation(B)
    lens, new = (None if x is None else x[order] for x in _lengths(case))
    tp = -(-case["max_len"] // P)
    pages = B * tp + 5                       # pages of a pool go to the sequences in any order
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dt)  # noqa: E731
    on_gpu = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()  # noqa: E731
    table = torch.randperm(pages, generator=g, device="cuda")[:B * tp].to(torch.int32).reshape(B, tp).contiguous()
    s = {"case": case, "table": table, "lens": on_gpu(lens), "lens_host": lens, "scale": D ** -0.5}
    if op == "pack":
        s["K"], s["V"] = (torch.zeros((pages, KV, P, D // 2 + D // 32), dtype=torch.uint8, device="cuda") for _ in range(2))
    elif op == "packed":
        s["K"], s["V"] = (_pool_fp4(*_nearest_fp4(torch.randn((pages, KV, P, D), generator=g, device="cuda")), is_v) for is_v in (False, True))
    else:
        s["K"] = normal(pages, KV, P, D)
        if op != "select":
            s["V"] = normal(pages, KV, P, D)
    if new is not None:
        s["new_host"], s["offsets"] = new, on_gpu(np.concatenate([[0], np.cumsum(new)]))
        total = int(new.sum())
        s["k_new"], s["v_new"], s["q"] = normal(total, KV, D), normal(total, KV, D), normal(total, H, D)
        s["seen"] = on_gpu(lens + case["ahead"])
        s["rotation"] = None
        if case["angles"]:
            at = torch.arange(case["max_len"] + case["ahead"], device="cuda", dtype=torch.float64)[:, None]
            angle = at * 10000.0 ** (-torch.arange(case["angles"] // 2, device="cuda", dtype=torch.float64) * 2 / case["angles"])
            s["rotation"] = torch.cat((angle.cos(), angle.sin()), -1).float()
        if op == "pack":
            s["k_rows"], s["v_rows"] = torch.zeros_like(s["k_new"]), torch.zeros_like(s["v_new"])
        elif case["track"]:
            s["positions"] = torch.full((B, KV, tp * P), -1, dtype=torch.int32, device="cuda")
        s["q_out"] = torch.zeros_like(s["q"])
    else:
        s["q"] = normal(B, H, D)
    if op == "packed" and case["spans"]:
        s["span_host"] = _span_lists(case, lens, rng)
        s["span"] = [on_gpu(a) for a in s["span_host"]]
    if op == "select":
        since = np.maximum(lens - max(case["fresh"], 1), 0)
        s["since"] = on_gpu(since) if case["fresh"] else None
        s["since_host"] = since
        s["bounds"] = _bounds_until(s, since)
        s["selected"] = torch.full((B, KV, case["budget"]), -1, dtype=torch.int32, device="cuda")
    if op == "chosen":
        # a page chosen by chance counts as well as one by its score: the first and the last are in it, short caches are listed whole
        here = torch.rand((B, KV, tp), generator=g, device="cuda")
        page = torch.arange(tp, device="cuda")
        count = (s["lens"].long()[:, None, None] + P - 1) // P
        here = here.masked_fill((page == 0) | (page == count - 1), 2.0).masked_fill(page >= count, -1.0)
        listed_pages = here.argsort(dim=-1, descending=True)[..., :case["budget"]]
        listed_pages = listed_pages.masked_fill(listed_pages >= count, 1 << 30).sort(-1).values
        listed_pages = listed_pages.masked_fill(listed_pages == 1 << 30, -1)
        s["selected"] = torch.nn.functional.pad(listed_pages, (0, case["budget"] - listed_pages.shape[-1]), value=-1).to(torch.int32).contiguous()
    if own:
        s["call"] = _handle(s)
    torch.cuda.synchronize()
    return s


def _bounds_until(s, since):
    """Bounds [pages, kv_heads, 2, head_dim] of the rows ahead of `since`, as earlier steps left them."""
    c = s["case"]
    P = c["page"]
    bounds = torch.zeros((s["K"].shape[0], c["kv_heads"], 2, c["head_dim"]), dtype=s["K"].dtype, device="cuda")
    start = torch.arange(s["table"].shape[1], device="cuda") * P
    rows = (torch.from_numpy(since).cuda()[:, None] - start).clamp(0, P)  # of every page
    for whole in (True, False):
        b, i = ((rows == P) if whole else (rows > 0) & (rows < P)).nonzero(as_tuple=True)
        if not b.numel():
            continue
        page = s["table"].long()[b, i]
        for at in range(0, page.numel(), 4096):
            x = s["K"][page[at:at + 4096]].float()
            out = torch.arange(P, device="cuda") >= rows[b, i][at:at + 4096, None]
            out = out[:, None, :, None]
            bounds[page[at:at + 4096], :, 0] = x.masked_fill(out, math.inf).amin(2).to(bounds.dtype)
            bounds[page[at:at + 4096], :, 1] = x.masked_fill(out, -math.inf).amax(2).to(bounds.dtype)
    return bounds


def _handle(s):
    """The prepared call that a program keeps for these tensors."""
    import paper_2404_09336_amd as span
    c = s["case"]
    if c["op"] == "select":
        return span.prepare_paged_select(s["q"], s["K"], s["bounds"], s["table"], s["lens"], c["budget"], sinks=c["sinks"], recent=c["recent"], since=s["since"],
                                         selected=s["selected"])
    cache = (s["K"], s["V"], s["table"])
    if c["op"] == "rotate":
        return span.prepare_paged_append_rotary(s["k_new"], s["v_new"], *cache, s["lens"], s["rotation"], s["offsets"], paired=c["paired"], q=s["q"], q_out=s["q_out"],
                                                seen=s["seen"], positions=s.get("positions"))
    if c["op"] == "pack":
        put = span.prepare_paged_append_fp4(s["k_new"], s["v_new"], *cache, s["lens"], s["offsets"], rotation=s["rotation"], paired=c["paired"], q=s["q"],
                                            q_out=s["q_out"], seen=s["seen"])
        get = span.prepare_paged_read_fp4(*cache, s["lens"], s["offsets"], k_rows=s["k_rows"], v_rows=s["v_rows"])
        return lambda: (put(), get())
    if c["op"] == "packed" and c["spans"]:
        off, st, en = s["span_host"]
        tokens = np.add.reduceat(en - st, off[:-1]).astype(np.int64)
        return span.prepare_paged_span_decode_attn_fp4(s["q"], *cache, *s["span"], s["scale"], tokens_per_seq=tokens)
    if c["op"] == "packed":
        return span.prepare_paged_decode_attn_fp4(s["q"], *cache, s["lens"], s["scale"], window=c["window"], sinks=c["sinks"])
    return span.prepare_paged_selected_decode_attn(s["q"], *cache, s["lens"], s["selected"], s["scale"])


def run(state):
    c = state["case"]
    if own:
        out = state["call"]()
    else:
        out = {"rotate": _plain_rotate, "pack": _plain_pack, "packed": _plain_packed, "select": _plain_select, "chosen": _plain_chosen}[c["op"]](state)
    if c["op"] == "rotate":
        return {"K": state["K"], "V": state["V"], "q": state["q_out"], **({"positions": state["positions"]} if c["track"] else {})}
    if c["op"] == "pack":
        return {"k": state["k_rows"], "v": state["v_rows"], "q": state["q_out"]}
    if c["op"] == "select":
        return {"bounds": state["bounds"], "selected": state["selected"]}
    return {"out": out}


def _new_rows(s):
    """Sequence and slot of every new row."""
    row = torch.arange(s["k_new"].shape[0], device="cuda")
    b = torch.searchsorted(s["offsets"][1:].long(), row, right=True)
    return b, s["lens"].long()[b] - s["offsets"].long()[b + 1] + row


def _turned(s, x, position):
    """Rows x [tokens, heads, head_dim] turned by the angles of their tokens' positions, in x's type."""
    c = s["case"]
    half = c["angles"] // 2
    if not half:
        return x.clone()
    cos, sin = (t.to(x.dtype)[:, None] for t in s["rotation"][position].split(half, dim=-1))
    one, two = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if c["paired"] else (slice(0, half), slice(half, 2 * half))
    y = x.clone()
    y[..., one] = x[..., one] * cos - x[..., two] * sin
    y[..., two] = x[..., one] * sin + x[..., two] * cos
    return y


def _plain_rotate(s):
    P = s["case"]["page"]
    b, p = _new_rows(s)
    position = (s["seen"].long() - s["lens"].long())[b] + p
    page = s["table"].long()[b, p // P]
    s["K"][page, :, p % P] = _turned(s, s["k_new"].float(), position).to(s["K"].dtype)
    s["V"][page, :, p % P] = s["v_new"]
    s["q_out"].copy_(_turned(s, s["q"].float(), position))
    if s["case"]["track"]:
        s["positions"][b, :, p] = position.to(torch.int32)[:, None].expand(-1, s["case"]["kv_heads"])


def _plain_pack(s):
    """(K in 64 bits, where a turned value lies next to the border between two of sixteen.)  The pages get the bytes, the rows the values."""
    c = s["case"]
    P, KV, D = c["page"], c["kv_heads"], c["head_dim"]
    b, p = _new_rows(s)
    position = (s["seen"].long() - s["lens"].long())[b] + p
    page, at = s["table"].long()[b, p // P], p % P
    for name, rows, x in (("K", "k_rows", _turned(s, s["k_new"].double(), position)), ("V", "v_rows", s["v_new"].double())):
        code, byte = _nearest_fp4(x)
        two = code[..., 0::2] | (code[..., 1::2] << 4)
        flat = s[name].view(-1, KV, P * (D // 2 + D // 32))
        group, r = (at // 16)[:, None], (at % 16)[:, None]
        i = torch.arange(D // 2, device="cuda")
        if name == "V":
            to = group * (8 * D) + (r // 4) * (2 * D) + (i // (D // 32)) * (D // 8) + (r % 4) * (D // 32) + i % (D // 32)
        else:
            to = group * (8 * D) + (i // 16) * 256 + r * 16 + i % 16
        j = torch.arange(D // 32, device="cuda")
        to = torch.cat((to, P * (D // 2) + group * (D // 2) + j * 16 + r), -1)
        head = torch.arange(KV, device="cuda")[None, :, None]
        flat[page[:, None, None], head, to[:, None, :]] = torch.cat((two, byte), -1)
        s[rows].copy_(_values_of(code, byte))
    s["q_out"].copy_(_turned(s, s["q"].float(), position))


def _attend(s, K, V, seen):
    """One token per sequence over rows [batch, kv_heads, positions, head_dim] in 32 bits, where `seen`."""
    c = s["case"]
    B, H, KV, D = c["batch"], c["heads"], c["kv_heads"], c["head_dim"]
    score = torch.matmul(s["q"].float().reshape(B, KV, H // KV, D), K.transpose(2, 3)) * s["scale"]
    score = score.masked_fill(~seen, float("-inf"))
    w = torch.exp(score - score.amax(-1, keepdim=True))
    w = w / w.sum(-1, keepdim=True)
    return torch.matmul(w, V).reshape(B, H, D)


def _plain_packed(s):
    c = s["case"]
    B, KV, D = c["batch"], c["kv_heads"], c["head_dim"]
    K, V = (_unpool_fp4(s[n][s["table"].long().reshape(-1)], n == "V").reshape(B, -1, KV, c["page"], D).transpose(1, 2).reshape(B, KV, -1, D) for n in ("K", "V"))
    p = torch.arange(K.shape[2], device="cuda")
    if c["spans"]:
        off, st, en = (x.long() for x in s["span"])
        b = torch.searchsorted(off[1:], torch.arange(st.numel(), device="cuda"), right=True)
        edge = torch.zeros((B, p.numel() + 1), dtype=torch.int32, device="cuda")
        one = torch.ones_like(b, dtype=torch.int32)
        edge.index_put_((b, st), one, accumulate=True).index_put_((b, en), -one, accumulate=True)
        seen = edge.cumsum(1)[:, :-1] > 0
    else:
        last = s["lens"].long()[:, None] - 1
        seen = p <= last
        if c["window"]:
            seen = seen & ((p > last - c["window"]) | (p < c["sinks"]))
    return _attend(s, K, V, seen[:, None, None])


def _plain_select(s):
    c = s["case"]
    B, KV, G, D, P = c["batch"], c["kv_heads"], c["heads"] // c["kv_heads"], c["head_dim"], c["page"]
    n = s["lens"].long()[:, None]
    since = s["since"].long()[:, None] if s["since"] is not None else n - 1
    start = torch.arange(s["table"].shape[1], device="cuda") * P
    b, i = ((start < n) & (start + P > since)).nonzero(as_tuple=True)            # pages with new rows
    page, first = s["table"].long()[b, i], start[i]
    p = first[:, None] + torch.arange(P, device="cuda")
    out = ~((p >= since[b]) & (p < n[b]))[:, None, :, None]
    rows, before = s["K"][page].float(), s["bounds"][page].float()
    kept = (first < since[b][:, 0])[:, None, None]                               # what is bounded already stays so
    lo = torch.minimum(rows.masked_fill(out, math.inf).amin(2), torch.where(kept, before[:, :, 0], math.inf))
    hi = torch.maximum(rows.masked_fill(out, -math.inf).amax(2), torch.where(kept, before[:, :, 1], -math.inf))
    s["bounds"][page] = torch.stack((lo, hi), 2).to(s["bounds"].dtype)
    # scores in 64 bits: neighbours in rank lie close together
    q = s["q"].double().reshape(B, KV, G, D)
    q = torch.cat((q.clamp(max=0).sum(2), q.clamp(min=0).sum(2)), -1)[..., None]  # meets (lo, hi)
    bound = s["bounds"][s["table"].long()].permute(0, 2, 1, 3, 4).reshape(B, KV, -1, 2 * D).double()
    score = torch.matmul(bound, q)[..., 0].float()
    count = (n + P - 1) // P
    always = (start < c["sinks"]) | (start + P > n - max(c["recent"], 1))
    score = score.masked_fill(always[:, None], math.inf).masked_fill((start >= n)[:, None], -math.inf)
    rank = score.sort(dim=-1, descending=True, stable=True).indices[..., :c["budget"]]
    none = 1 << 30
    rank = rank.masked_fill(rank >= count[:, None], none).sort(-1).values
    s["selected"].fill_(-1)
    s["selected"][..., :rank.shape[-1]] = rank.masked_fill(rank == none, -1)


def _plain_chosen(s):
    c = s["case"]
    B, KV, P, D = c["batch"], c["kv_heads"], c["page"], c["head_dim"]
    chosen = s["selected"].long()
    page = torch.gather(s["table"].long()[:, None].expand(-1, KV, -1), 2, chosen.clamp(min=0))
    head = torch.arange(KV, device="cuda")[None, :, None]
    K, V = (s[x][page, head].reshape(B, KV, -1, D).float() for x in ("K", "V"))
    p = chosen[..., None] * P + torch.arange(P, device="cuda")
    seen = (chosen[..., None] >= 0) & (p < s["lens"].long()[:, None, None, None])
    return _attend(s, K, V, seen.reshape(B, KV, 1, -1))


def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    B, H, KV, D, P = c["batch"], c["heads"], c["kv_heads"], c["head_dim"], c["page"]
    lens, new = _lengths(c)
    row4 = D // 2 + D // 32
    if c["op"] == "rotate":
        return {"bytes": int(new.sum()) * (2 * (H + 2 * KV) * D * e + 4 * c["angles"] + (4 * KV if c["track"] else 0)), "flops": int(new.sum()) * 3 * (H + KV) * c["angles"]}
    if c["op"] == "pack":  # (read, packed, unpacked)
        return {"bytes": int(new.sum()) * ((2 * H + 4 * KV) * D * e + 4 * KV * row4 + 4 * c["angles"]), "flops": int(new.sum()) * 3 * (H + KV) * c["angles"]}
    if c["op"] == "packed":
        seen = np.minimum(lens, c["window"] + c["sinks"]) if c["window"] else lens
        if c["spans"]:  # (the beginning, the recent positions and a sixth of what is between)
            seen = np.minimum(lens, 112 + np.maximum(lens - 112, 0) // 6)
        seen = int(seen.sum())
        return {"bytes": seen * KV * 2 * row4 + B * H * D * (e + 4), "flops": 4 * H * D * seen}
    pages = -(-lens // P)
    if c["op"] == "select":
        scored, rows = int(pages[pages > c["budget"]].sum()), int(np.minimum(lens, max(c["fresh"], 1)).sum())
        return {"bytes": KV * (scored * 2 * D * e + rows * D * e + 4 * B * c["budget"]) + B * H * D * e, "flops": 4 * KV * D * scored}
    seen = int(np.minimum(lens, c["budget"] * P).sum())
    return {"bytes": seen * KV * 2 * D * e + 4 * B * KV * c["budget"] + B * H * D * (e + 4), "flops": 4 * H * D * seen}


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    B, P, H, KV, D = c["batch"], c["page"], c["heads"], c["kv_heads"], c["head_dim"]
    G = H // KV
    table, lens = s["table"].cpu().numpy().astype(np.int64), s["lens_host"]
    if c["op"] in ("rotate", "pack"):
        half = c["angles"] // 2
        place = np.concatenate([np.arange(n - t, n) for n, t in zip(lens, s["new_host"])])
        owner = np.repeat(np.arange(B), s["new_host"])

        def turned(x):
            """As a product of complex numbers."""
            x = x.double().clone()
            if half:
                angle = s["rotation"][torch.from_numpy(place + c["ahead"]).cuda()].double()
                turn = torch.complex(angle[:, :half].contiguous(), angle[:, half:].contiguous())[:, None]
                part = x[..., :2 * half]
                if c["paired"]:
                    z = torch.view_as_complex(part.unflatten(-1, (half, 2)).contiguous()) * turn
                    x[..., :2 * half] = torch.view_as_real(z).flatten(-2)
                else:
                    z = torch.complex(part[..., :half].contiguous(), part[..., half:].contiguous()) * turn
                    x[..., :2 * half] = torch.cat((z.real, z.imag), -1)
            return x

        if c["op"] == "rotate":
            page, at = (torch.from_numpy(x).cuda() for x in (table[owner, place // P], place % P))
            K, V = s["K"].double(), s["V"].double()
            K[page, :, at] = turned(s["k_new"])
            V[page, :, at] = s["v_new"].double()
            return {"K": K, "V": V, "q": turned(s["q"]), **({"positions": None} if c["track"] else {})}

        def nearest(x):
            """By the borders between neighbouring values; a value on a border goes to the one with an even number."""
            x = x.unflatten(-1, (-1, 32))
            most = x.abs().amax(-1, keepdim=True)
            unit = torch.exp2(torch.ceil(torch.log2(most / 7).clamp(min=-126)))
            unit = torch.where(most > 7 * unit, unit * 2, torch.where(most <= 3.5 * unit, unit / 2, unit))  # (the logarithm may be off next to a whole number)
            y = (x.abs() / unit).contiguous()
            border = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64, device=x.device)
            number = torch.searchsorted(border, y)
            tie = (y == border[number.clamp(max=6)]) & (number % 2 == 1)
            value = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 6], dtype=torch.float64, device=x.device)[number + tie.long()]
            return (torch.copysign(value, x) * unit).flatten(-2)

        return {"k": nearest(turned(s["k_new"])), "v": nearest(s["v_new"].double()), "q": turned(s["q"])}
    if c["op"] == "select":
        bounds = s["bounds"].double()
        for b, n in enumerate(lens):
            since = int(s["since_host"][b])
            for i in range(since // P, -(-int(n) // P)):
                a, z = max(since - i * P, 0), min(int(n) - i * P, P)
                new = s["K"][table[b, i], :, a:z].double()
                old = bounds[table[b, i]][:, :, None][:, :, :0 if a == 0 else 1]
                bounds[table[b, i], :, 0] = torch.cat((old[:, 0], new), 1).min(1).values
                bounds[table[b, i], :, 1] = torch.cat((old[:, 1], new), 1).max(1).values
        return {"bounds": bounds, "selected": None}
    packed = c["op"] == "packed"
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    number = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device="cuda")
    d = torch.arange(D, device="cuda")

    def rows(pool, page, h, at, is_v):
        """Rows of one head in 64 bits."""
        page, at = torch.from_numpy(page).cuda(), torch.from_numpy(at).cuda()
        if not packed:
            return pool[page, h, at].double()
        flat = pool.view(pool.shape[0], KV, -1)
        group, r = (at // 16)[:, None], (at % 16)[:, None]
        if is_v:  # fours of rows, sixteenths of the channels, rows
            byte = ((group * 4 + r // 4) * 16 + d // (D // 16)) * (D // 8) + r % 4 * (D // 32) + d % (D // 16) // 2
        else:     # blocks of 32 channels, rows
            byte = ((group * (D // 32) + d // 32) * 16 + r) * 16 + d % 32 // 2
        two = flat[page[:, None], h, byte].long()
        power = flat[page[:, None], h, P * D // 2 + (group * (D // 32) + d // 32) * 16 + r].double() - 127
        return number[torch.where(d % 2 == 1, two // 16, two % 16)] * torch.exp2(power)

    for b, n in enumerate(lens):
        for h in range(KV):
            if c["op"] == "chosen":
                chosen = s["selected"][b, h].cpu().numpy().astype(np.int64)
                p = (chosen[chosen >= 0][:, None] * P + np.arange(P)).reshape(-1)
                p = p[p < n]
            elif c["spans"]:
                off, st, en = s["span_host"]
                p = np.concatenate([np.arange(x, y) for x, y in zip(st[off[b]:off[b + 1]], en[off[b]:off[b + 1]])]).astype(np.int64)
            else:
                p = np.arange(n)
                if c["window"]:
                    p = p[(p >= n - c["window"]) | (p < c["sinks"])]
            page, at = table[b, p // P], p % P
            k, v = rows(s["K"], page, h, at, False), rows(s["V"], page, h, at, True)
            w = torch.softmax(s["q"][b, h * G:(h + 1) * G].double() @ k.T.contiguous() * s["scale"], -1)
            out[b, h * G:(h + 1) * G] = w @ v
    return {"out": out}
