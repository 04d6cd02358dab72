"""The operators on a cache in pages as cases that can be timed and compared: `run` computes them from elementary torch operations in 32 bits
(`own` false) or makes the framework's calls (`own` true).

Keys of a case
  op        "append"  rows of new tokens into the pages                        (paged_append)
            "decode"  one token per sequence over its cache                    (paged_decode_attn; paged_span_decode_attn with `spans`)
            "prompt"  the new tokens of every sequence over its cache, causal  (paged_prompt_attn)
            "evict"   the cache cut down to a budget                           (paged_evict)
  dtype     "f32" | "f16" | "bf16"
  batch, heads, kv_heads, head_dim, page
  min_len, max_len   cached positions of a sequence, the new tokens among them, drawn uniformly
  min_new, max_new   "append", "prompt": new tokens of a sequence, drawn uniformly, at most its cached positions
  window, sinks      "decode", "prompt": a token sees the last `window` positions up to its own (0: all) and the first `sinks`
  spans              "decode": intervals of a sequence (0: no span lists)
  weights            "decode": the attention weights are added up per cached position
  track              "append": the positions of the rows are noted for an eviction
  budget, recent     "evict": slots that stay; the last `recent` positions and the first `sinks` stay in any case
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
        # what every decode step does first: one row per sequence and head into its page, the positions noted for a later eviction
        _case("append-step-f16", "append", "f16", 64, (32, 8), 128, 16, (400, 4096), min_new=1, max_new=1, track=True),
        # prompts of a served batch going into the cache, as many KV heads as query heads
        _case("append-prompts-bf16", "append", "bf16", 16, (32, 32), 128, 64, (100, 4096), min_new=100, max_new=4096, track=False),
        # the smallest call anybody makes: latency and launch cost only
        _case("decode-tiny-f32", "decode", "f32", 1, (4, 4), 64, 16, (256, 256), window=0, sinks=0, spans=0, weights=False),
        # a served batch, four query heads per KV head, ragged
        _case("decode-batch-bf16", "decode", "bf16", 64, (32, 8), 128, 64, (512, 4096), window=0, sinks=0, spans=0, weights=False),
        # long conversations of a model with a sliding window whose first four tokens stay visible
        _case("decode-window-f16", "decode", "f16", 32, (32, 8), 128, 16, (700, 16384), window=1024, sinks=4, spans=0, weights=False),
        # four long documents whose positions are weighed for an eviction
        _case("decode-weights-bf16", "decode", "bf16", 4, (32, 8), 128, 256, (8000, 32768), window=0, sinks=0, spans=0, weights=True),
        # self-selected spans (an instruction, a few line ranges, the recent tokens) of 16 articles, one query head per KV head
        _case("decode-span-f16", "decode", "f16", 16, (32, 32), 128, 16, (2048, 4096), window=0, sinks=0, spans=5, weights=False),
        # one long prompt: the largest work
        _case("prompt-long-bf16", "prompt", "bf16", 1, (32, 8), 128, 64, (8192, 8192), min_new=8192, max_new=8192, window=0, sinks=0),
        # chunks of prompts behind a cached beginning, ragged, sliding window and sinks
        _case("prompt-window-f16", "prompt", "f16", 6, (32, 8), 128, 16, (1500, 4100), min_new=333, max_new=1500, window=1024, sinks=4),
        # short prompts of a small model in fp32
        _case("prompt-short-f32", "prompt", "f32", 3, (12, 4), 64, 16, (77, 301), min_new=77, max_new=301, window=0, sinks=0),
        # a served batch that outgrew its budget by an eighth at most
        _case("evict-batch-f16", "evict", "f16", 16, (32, 8), 128, 16, (4096, 4608), budget=4096, sinks=4, recent=256),
        # long caches cut down hard, some sequences below the budget
        _case("evict-deep-bf16", "evict", "bf16", 5, (16, 16), 64, 64, (900, 12001), budget=2048, sinks=4, recent=100),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: batch 1 .. 64, 1 .. 32768 cached positions, caches up to 1 GiB, prompts up to the work of the largest listed one."""
    op = rng.choice(["append", "decode", "decode", "decode", "decode", "prompt", "prompt", "evict", "evict"])
    dtype = rng.choice(["f16", "bf16", "bf16", "f32"])
    heads = rng.choice([(32, 8), (32, 32), (16, 2), (12, 4), (14, 2), (5, 5), (8, 1), (16, 1), (6, 3)])
    head_dim = rng.choice([128, 128, 64])
    page = rng.choice([16, 32, 64, 256])
    batch, top = _log_int(rng, 1, 64), _log_int(rng, 16, 32768 if op == "decode" else 8192)
    row = 2 * heads[1] * head_dim * (4 if dtype == "f32" else 2)
    bound = 1 << 29 if op in ("decode", "append") else 1 << 28
    while batch * top * row > bound or (op == "prompt" and batch * heads[0] * top * top * head_dim > 1 << 38):
        batch, top = (max(batch // 2, 1), top) if batch > 1 else (1, top // 2)
    low = max(1, int(top * rng.uniform(0.1, 1.0)))
    more = {}
    if op in ("append", "prompt"):
        most = 1 if op == "append" and rng.random() < 0.5 else _log_int(rng, 1, top)
        more = {"min_new": max(1, int(most * rng.uniform(0.2, 1.0))), "max_new": most}
    if op == "append":
        more["track"] = rng.random() < 0.5
    if op in ("decode", "prompt"):
        windowed = rng.random() < 0.5
        more.update(window=_log_int(rng, 1, top) if windowed else 0, sinks=rng.choice([0, 1, 4, 17, 64]) if windowed else 0)
    if op == "decode":
        more.update(spans=rng.choice([0, 1, 7, 40]) if not more["window"] else 0, weights=rng.random() < 0.4)
    if op == "evict":
        budget = max(8, int(top * rng.uniform(0.2, 1.0)))
        more = {"budget": budget, "sinks": rng.choice([0, 1, 4]), "recent": int((budget - 4) * rng.uniform(0.0, 1.0))}
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


def prepare(case, seed):
    torch.cuda.synchronize()
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, B, H, KV, D, P = _DTYPES[case["dtype"]], case["batch"], case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    rng = np.random.default_rng(seed)
    order = rng.permutation(B)
    lens, new = (None if x is None else x[order] for x in _lengths(case))
    tp = -(-case["max_len"] // P)
    pages = B * tp + 5                       # pages of a pool go to the sequences in any order
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dt)  # noqa: E731
    on_gpu = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()  # noqa: E731
    table = torch.randperm(pages, generator=g, device="cuda")[:B * tp].to(torch.int32).reshape(B, tp).contiguous()
    s = {"case": case, "K": normal(pages, KV, P, D), "V": normal(pages, KV, P, D), "table": table, "lens": on_gpu(lens), "lens_host": lens, "scale": D ** -0.5}
    op = case["op"]
    if new is not None:
        s["new_host"], s["offsets"] = new, on_gpu(np.concatenate([[0], np.cumsum(new)]))
        total = int(new.sum())
        if op == "append":
            s["k_new"], s["v_new"] = normal(total, KV, D), normal(total, KV, D)
            if case["track"]:
                s["seen"] = on_gpu(lens + 1000)
                s["positions"] = torch.full((B, KV, tp * P), -1, dtype=torch.int32, device="cuda")
        else:
            s["q"] = normal(total, H, D)
    if op == "decode":
        s["q"] = normal(B, H, D)
        if case["spans"]:
            s["span_host"] = _span_lists(case, lens, rng)
            s["span"] = [on_gpu(a) for a in s["span_host"]]
        if case["weights"]:
            s["weights"] = torch.rand((B, KV, tp * P), generator=g, device="cuda") / 1000
    if op == "evict":
        # what a decode loop has added up: skewed, and nothing yet for some of the last tokens
        w = torch.rand((B, KV, tp * P), generator=g, device="cuda").pow(4)
        slot = torch.arange(tp * P, device="cuda")
        s["weights"] = w.masked_fill(slot >= s["lens"][:, None, None] - 3, 0.0)
        # slots hold ascending positions but for some that an earlier eviction filled
        ahead = torch.rand((B, KV, tp * P), generator=g, device="cuda").mul(40).long() * (torch.rand((B, KV, tp * P), generator=g, device="cuda") < 0.1)
        s["positions"] = (slot + ahead).argsort(dim=-1, stable=True).to(torch.int32)
        s["weights_out"], s["positions_out"] = torch.zeros_like(s["weights"]), torch.full_like(s["positions"], -1)
        s["new_lens"] = torch.zeros_like(s["lens"])
    if own:
        s["call"] = _handle(s)
    torch.cuda.synchronize()
    return s


def _handle(s):
    """The prepared call that a program keeps for these tensors."""
    import paper_2404_09336_amd as span
    c = s["case"]
    cache = (s["K"], s["V"], s["table"])
    if c["op"] == "append":
        track = {"positions": s["positions"], "seen": s["seen"]} if c["track"] else {}
        return span.prepare_paged_append(s["k_new"], s["v_new"], *cache, s["lens"], s["offsets"], **track)
    if c["op"] == "decode" and c["spans"]:
        off, st, en = s["span_host"]
        tokens = np.add.reduceat(en - st, off[:-1]).astype(np.int64)
        return span.prepare_paged_span_decode_attn(s["q"], *cache, *s["span"], s["scale"], weights=s.get("weights"), tokens_per_seq=tokens)
    if c["op"] == "decode":
        return span.prepare_paged_decode_attn(s["q"], *cache, s["lens"], s["scale"], window=c["window"], sinks=c["sinks"], weights=s.get("weights"))
    if c["op"] == "prompt":
        return span.prepare_paged_prompt_attn(s["q"], *cache, s["lens"], s["offsets"], s["scale"], window=c["window"], sinks=c["sinks"])
    return span.prepare_paged_evict(*cache, s["lens"], s["weights"], c["budget"], positions=s["positions"], sinks=c["sinks"], recent=c["recent"],
                                    weights_out=s["weights_out"], positions_out=s["positions_out"], new_lens=s["new_lens"])


def run(state):
    c = state["case"]
    if own:
        out = state["call"]()
    else:
        out = {"append": _plain_append, "decode": _plain_decode, "prompt": _plain_prompt, "evict": _plain_evict}[c["op"]](state)
    if c["op"] == "append":
        return {"K": state["K"], "V": state["V"], **({"positions": state["positions"]} if c["track"] else {})}
    if c["op"] == "evict":
        return {"K": state["K"], "V": state["V"], "weights": state["weights_out"], "positions": state["positions_out"], "lens": state["new_lens"]}
    return {"out": out, **({"weights": state["weights"]} if c.get("weights") else {})}


def _new_rows(s):
    """Sequence and position of every new row."""
    row = torch.arange(s["k_new" if "k_new" in s else "q"].shape[0], device="cuda")
    b = torch.searchsorted(s["offsets"][1:].long(), row, right=True)
    return b, s["lens"].long()[b] - s["offsets"].long()[b + 1] + row


def _plain_append(s):
    P = s["case"]["page"]
    b, p = _new_rows(s)
    page = s["table"].long()[b, p // P]
    s["K"][page, :, p % P] = s["k_new"]
    s["V"][page, :, p % P] = s["v_new"]
    if s["case"]["track"]:
        s["positions"][b, :, p] = (s["seen"][b] - s["lens"][b] + p).to(torch.int32)[:, None].expand(-1, s["case"]["kv_heads"])


def _rows(s, pool):
    """The caches as [batch, kv_heads, positions, head_dim] in fp32."""
    c = s["case"]
    x = s[pool][s["table"].long()].permute(0, 2, 1, 3, 4)
    return x.reshape(c["batch"], c["kv_heads"], -1, c["head_dim"]).float()


def _visible(s, last, p):
    """Whether a token at position `last` sees position p."""
    c = s["case"]
    seen = p <= last
    return seen & ((p > last - c["window"]) | (p < c["sinks"])) if c["window"] else seen


def _plain_decode(s):
    c = s["case"]
    B, H, KV, D = c["batch"], c["heads"], c["kv_heads"], c["head_dim"]
    K, V = _rows(s, "K"), _rows(s, "V")
    p = torch.arange(K.shape[2], device="cuda")
    if c["spans"]:
        off, st, en = (x.long() for x in s["span"])
        b = torch.searchsorted(off[1:], torch.arange(st.numel(), device="cuda"), right=True)
        edge = torch.zeros((B, p.numel() + 1), dtype=torch.int32, device="cuda")
        one = torch.ones_like(b, dtype=torch.int32)
        edge.index_put_((b, st), one, accumulate=True).index_put_((b, en), -one, accumulate=True)
        seen = edge.cumsum(1)[:, :-1] > 0
    else:
        seen = _visible(s, s["lens"].long()[:, None] - 1, p)
    score = torch.matmul(s["q"].float().reshape(B, KV, H // KV, D), K.transpose(2, 3)) * s["scale"]
    score = score.masked_fill(~seen[:, None, None], float("-inf"))
    w = torch.exp(score - score.amax(-1, keepdim=True))
    w = w / w.sum(-1, keepdim=True)
    if c["weights"]:
        s["weights"] += w.sum(2)
    return torch.matmul(w, V).reshape(B, H, D)


def _plain_prompt(s):
    c = s["case"]
    B, H, KV, D = c["batch"], c["heads"], c["kv_heads"], c["head_dim"]
    K, V = _rows(s, "K"), _rows(s, "V")
    b, last = _new_rows(s)
    most = int(s["new_host"].max())
    i = last - (s["lens"].long() - (s["offsets"][1:] - s["offsets"][:-1]).long())[b]  # token of its sequence
    q = torch.zeros((B, most, H, D), device="cuda")
    q[b, i] = s["q"].float()
    at = torch.zeros((B, most), dtype=torch.long, device="cuda")
    at[b, i] = last
    q = q.reshape(B, most, KV, H // KV, D).permute(0, 2, 3, 1, 4).reshape(B, KV, -1, D)
    score = torch.matmul(q, K.transpose(2, 3)).reshape(B, KV, H // KV, most, -1).mul_(s["scale"])
    seen = _visible(s, at[:, :, None], torch.arange(K.shape[2], device="cuda"))
    score.masked_fill_(~seen[:, None, None], float("-inf"))
    w = score.sub_(score.amax(-1, keepdim=True)).exp_()
    w /= w.sum(-1, keepdim=True)
    out = torch.matmul(w.reshape(B, KV, -1, w.shape[-1]), V).reshape(B, H, most, D)
    return out.transpose(1, 2)[b, i].to(s["q"].dtype)


def _plain_evict(s):
    c = s["case"]
    B, KV, P, keep = c["batch"], c["kv_heads"], c["page"], c["budget"]
    slot = torch.arange(s["weights"].shape[2], device="cuda")
    n = s["lens"].long()[:, None, None]
    held = slot < n                                                   # slots in use
    pos = s["positions"]
    last = pos.masked_fill(~held, -1).amax(-1, keepdim=True)
    safe = (pos < c["sinks"]) | (pos > last - c["recent"])
    rank = s["weights"].masked_fill(safe, float("inf")).masked_fill(~held, float("-inf")).sort(dim=-1, descending=True, stable=True).indices
    stays = torch.zeros_like(safe)
    stays.scatter_(2, rank[..., :keep], True)
    stays &= held
    cut = n > keep
    to, of = ((~stays & held & cut & (slot < keep)).nonzero(), (stays & cut & (slot >= keep)).nonzero())  # equally many of a head, both ascending
    b, h, d, f = to[:, 0], to[:, 1], to[:, 2], of[:, 2]
    table = s["table"].long()
    for name in ("K", "V"):
        s[name][table[b, d // P], h, d % P] = s[name][table[b, f // P], h, f % P]
    left = n.clamp(max=keep)
    for name, none in (("weights", 0.0), ("positions", -1)):
        out = s[name].clone()
        out[b, h, d] = s[name][b, h, f]
        s[name + "_out"].copy_(torch.where(held, out.masked_fill(slot >= left, none), s[name + "_out"]))
    s["new_lens"].copy_(left.reshape(-1))


def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    B, H, KV, D = c["batch"], c["heads"], c["kv_heads"], c["head_dim"]
    lens, new = _lengths(c)
    if c["op"] == "append":
        return {"bytes": int(new.sum()) * KV * (4 * D * e + (4 if c["track"] else 0)), "flops": 0}
    if c["op"] == "decode":
        seen = np.minimum(lens, c["window"] + c["sinks"]) if c["window"] else lens
        if c["spans"]:  # (the beginning, the recent positions and a sixth of what is between)
            seen = np.minimum(lens, 112 + np.maximum(lens - 112, 0) // 6)
        seen = int(seen.sum())
        return {"bytes": seen * KV * (2 * D * e + (8 if c["weights"] else 0)) + B * H * D * (e + 4), "flops": 4 * H * D * seen}
    if c["op"] == "prompt":
        pairs = 0
        for n, t in zip(lens.tolist(), new.tolist()):
            at = np.arange(n - t, n) + 1  # positions up to a token's own
            pairs += int((np.minimum(at, c["window"] + c["sinks"]) if c["window"] else at).sum())
        return {"bytes": 2 * int(new.sum()) * H * D * e + 2 * int(lens.sum()) * KV * D * e, "flops": 4 * H * D * pairs}
    out = np.maximum(lens - c["budget"], 0)  # rows that go, and as many slots past the budget: protected ones move, the others by chance
    moved = np.minimum(np.minimum(out, c["recent"]) + np.maximum(out - c["recent"], 0) * (c["budget"] / lens), c["budget"])
    return {"bytes": int(KV * (moved * 4 * D * e + 16 * lens).sum()), "flops": 0}


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    P, KV, G = c["page"], c["kv_heads"], c["heads"] // c["kv_heads"]
    table, lens = s["table"].cpu().numpy().astype(np.int64), s["lens_host"]
    if c["op"] == "append":
        first, K, V = 0, s["K"].double(), s["V"].double()
        for b, t in enumerate(s["new_host"]):
            for p0 in range(int(lens[b] - t), int(lens[b])):
                if p0 % P and p0 > lens[b] - t:
                    continue
                p1 = min((p0 // P + 1) * P, int(lens[b]))
                rows = slice(first + p0 - int(lens[b] - t), first + p1 - int(lens[b] - t))
                K[table[b, p0 // P], :, p0 % P:p0 % P + p1 - p0] = s["k_new"][rows].transpose(0, 1).double()
                V[table[b, p0 // P], :, p0 % P:p0 % P + p1 - p0] = s["v_new"][rows].transpose(0, 1).double()
            first += int(t)
        return {"K": K, "V": V, **({"positions": None} if c["track"] else {})}

    def row(b, p):  # pool rows of positions p of sequence b
        return torch.from_numpy(table[b, p // P]).cuda(), torch.from_numpy(p % P).cuda()

    def attend(b, h, p, queries, limit):
        """Weights [queries, positions] and outputs of kv head h; `limit`: what each query sees of the positions, or None."""
        page, at = row(b, p)
        score = queries.double() @ s["K"][page, h, at].double().T.contiguous() * s["scale"]
        if limit is not None:
            score[~limit] = -math.inf
        w = torch.softmax(score, -1)
        return w, w @ s["V"][page, h, at].double()

    if c["op"] == "decode":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        weights = s["weights"].double() if c["weights"] else None
        for b, n in enumerate(lens):
            p = np.arange(n)
            if c["spans"]:
                off, st, en = s["span_host"]
                p = np.concatenate([np.arange(x, y) for x, y in zip(st[off[b]:off[b + 1]], en[off[b]:off[b + 1]])])
            elif c["window"]:
                p = p[(p >= n - c["window"]) | (p < c["sinks"])]
            for h in range(KV):
                w, out[b, h * G:(h + 1) * G] = attend(b, h, p, s["q"][b, h * G:(h + 1) * G], None)
                if weights is not None:
                    weights[b, h, torch.from_numpy(p).cuda()] += w.sum(0)
        return {"out": out, **({"weights": weights} if c["weights"] else {})}
    if c["op"] == "prompt":
        out, first = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"), 0
        for b, t in enumerate(s["new_host"]):
            n, t = int(lens[b]), int(t)
            p = np.arange(n)
            own_at = np.arange(n - t, n)[:, None]
            limit = p <= own_at
            if c["window"]:
                limit &= (own_at - p < c["window"]) | (p < c["sinks"])
            limit = torch.from_numpy(limit).cuda()
            for h in range(KV):
                for g in range(h * G, (h + 1) * G):
                    out[first:first + t, g] = attend(b, h, p, s["q"][first:first + t, g], limit)[1]
            first += t
        return {"out": out}
    K, V = s["K"].double(), s["V"].double()
    weights, positions = s["weights"].cpu().numpy(), s["positions"].cpu().numpy()
    w_out = np.zeros(weights.shape)
    to_page, to_at, of_page, of_at, head = [], [], [], [], []
    for b, n in enumerate(lens):
        n, keep = int(n), c["budget"]
        for h in range(KV):
            w, pos = weights[b, h, :n], positions[b, h, :n]
            if n <= keep:
                w_out[b, h, :n] = w
                continue
            safe = (pos < c["sinks"]) | (pos > pos.max() - c["recent"])
            order = np.lexsort((np.arange(n), -w.astype(np.float64), ~safe))   # protected ones first, then by weight, then by slot
            stays = np.sort(order[:keep])
            holes = np.setdiff1d(np.arange(keep), stays)
            movers = stays[stays >= keep]
            w_out[b, h, :keep] = w[:keep]
            w_out[b, h, holes] = w[movers]
            to_page.append(table[b, holes // P])
            to_at.append(holes % P)
            of_page.append(table[b, movers // P])
            of_at.append(movers % P)
            head.append(np.full(holes.size, h))
    if head:
        tp, ta, fp, fa, hd = (torch.from_numpy(np.concatenate(x)).cuda() for x in (to_page, to_at, of_page, of_at, head))
        K[tp, hd, ta] = K[fp, hd, fa]
        V[tp, hd, ta] = V[fp, hd, fa]
    return {"K": K, "V": V, "weights": torch.from_numpy(w_out), "positions": None, "lens": None}
