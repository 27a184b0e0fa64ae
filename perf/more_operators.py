"""More operators around the paged 8-bit cache, as cases to be timed.

- tree: the mask of a tree of drafted tokens, and attention of those tokens over the cache by it.
- weights: how much attention every cached token gets from a step's queries, added to what it had before.
- select: which tokens of every sequence and head stay when a cache is cut down to a budget.
- keep: moving the tokens that stay together, a drafted path that was accepted or a selection, scales and all.

Head counts and sizes are those of the repository's workloads (4096 and 8192 channels in heads of 128, sequences of
1000, 4096, 8192 and up to 131072 tokens) and generic ones around them.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 16                                   # tokens per scale
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # One sequence, 16 drafted tokens to verify, a short cache: latency.
        dict(name="tree_step", kind="tree", batch=1, len=1001, spread=0.0, new=16, ragged=False, page=64,
             hq=64, hkv=8, d=128, fmt="int8", dtype="bf16", window=0),
        # A serving batch with trees of up to 26 tokens, a kv head per query head, the e4m3 cache.
        dict(name="tree_batch", kind="tree", batch=16, len=4096, spread=0.9, new=26, ragged=True, page=16,
             hq=32, hkv=32, d=128, fmt="e4m3", dtype="f16", window=0),
        # Two long documents with trees of 64 tokens.
        dict(name="tree_long", kind="tree", batch=2, len=65536, spread=0.2, new=64, ragged=False, page=256,
             hq=64, hkv=8, d=128, fmt="int8", dtype="bf16", window=0),
        # Heads of 64 channels, fp32, a sliding window, up to 7 tokens in a tree.
        dict(name="tree_window", kind="tree", batch=8, len=3001, spread=0.7, new=7, ragged=True, page=32,
             hq=32, hkv=4, d=64, fmt="int8", dtype="f32", window=2000),
        # One sequence, the step's one token: latency.
        dict(name="weights_step", kind="weights", batch=1, len=1001, spread=0.0, new=1, ragged=False, page=64,
             hq=64, hkv=8, d=128, fmt="int8", dtype="bf16", window=0, before=True),
        # Every step of a serving batch, a kv head per query head.
        dict(name="weights_batch", kind="weights", batch=64, len=4096, spread=0.95, new=1, ragged=False, page=16,
             hq=32, hkv=32, d=128, fmt="e4m3", dtype="f16", window=0, before=True),
        # What the last 64 tokens of two prompts look at, before the prompts' caches are cut down.
        dict(name="weights_prompt", kind="weights", batch=2, len=32768, spread=0.3, new=64, ragged=False, page=64,
             hq=64, hkv=8, d=128, fmt="int8", dtype="bf16", window=0, before=False),
        # A short sequence, half of it kept: latency.
        dict(name="select_step", kind="select", batch=1, len=1001, spread=0.0, hkv=8, keep=500, first=4, recent=64),
        # Four long documents down to 4096 tokens.
        dict(name="select_long", kind="select", batch=4, len=131072, spread=0.2, hkv=8, keep=4096, first=4, recent=512),
        # The accepted paths (up to 6 of 16 drafted tokens) of a batch, moved behind the sequences in place.
        dict(name="keep_path", kind="keep", batch=16, len=1000, spread=0.8, new=16, kept=6, each=False, in_place=True,
             page=64, hkv=8, d=128, fmt="int8", dtype="bf16"),
        # Eight prompts down to 2047 tokens a head, into new pages.
        dict(name="keep_copy", kind="keep", batch=8, len=8192, spread=0.5, new=0, kept=2047, each=True, in_place=False,
             page=16, hkv=32, d=128, fmt="e4m3", dtype="f16"),
        # Two long documents down to 16384 tokens a head, in their own pages.
        dict(name="keep_in_place", kind="keep", batch=2, len=65536, spread=0.2, new=0, kept=16384, each=True,
             in_place=True, page=256, hkv=8, d=128, fmt="int8", dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choice(["tree", "tree", "tree", "weights", "weights", "select", "keep", "keep"])
    hkv = rng.choice([1, 2, 4, 8, 32])
    c = dict(kind=kind, batch=_log(rng, 1, 64), spread=rng.choice([0.0, 0.5, 0.95]), hkv=hkv)
    if kind == "select":
        most = 4 * 131072 * 8 // (hkv * c["batch"])             # weights in all
        c["len"] = _log(rng, 20, min(most, 131072))
        c["keep"] = _log(rng, 16, min(c["len"], 16384))
        c["first"] = rng.choice([0, 4]) if c["keep"] > 8 else 0
        c["recent"] = rng.randint(0, c["keep"] // 2)
        return c
    c.update(page=rng.choice([16, 32, 48, 64, 128, 256]), d=rng.choice([64, 128]), fmt=rng.choice(["int8", "e4m3"]),
             dtype=rng.choice(["bf16", "f16", "bf16", "f16", "f32"]))
    most = 2 * 65536 * 8 * 128 // (hkv * c["d"] * c["batch"])    # cached channels in all
    c["len"] = _log(rng, 64, max(64, min(most, 65536)))
    if kind == "keep":
        c["in_place"], c["each"] = rng.random() < 0.5, rng.random() < 0.7
        c["new"] = 0 if c["each"] else rng.randint(2, 48)
        # (rows read back in 32 bits count for more)
        top = min(c["len"], 2 * 16384 * 8 * 128 // (hkv * c["d"] * c["batch"] * (2 if c["dtype"] == "f32" else 1)))
        c["kept"] = _log(rng, 1, max(1, top)) if c["each"] else rng.randint(1, min(8, c["new"]))
        return c
    c["hq"] = hkv * rng.choice([1, 1, 2, 4, 8] if hkv < 32 else [1, 2])
    c["ragged"] = rng.random() < 0.5
    c["window"] = rng.choice([0, 0, 0, _log(rng, 16, 4096)])
    c["new"] = rng.randint(2, 16) if rng.random() < 0.5 else _log(rng, 9, 64)
    if kind == "weights":
        c["new"] = rng.choice([1, 1, 1, c["new"]])
        c["before"] = rng.random() < 0.7
    # no more score entries than the listed trees have
    c["new"] = max(1, min(c["new"], 2 * 64 * 64 * 65536 // (c["batch"] * c["hq"] * c["len"])))
    return c


# ---------------------------------------------------------------- sizes
def _spread(n, i, most, by):
    return max(1, round(most * (1.0 - by * ((i * 0.6180339887498949) % 1.0)))) if n else 0


def _totals(case):
    """Tokens of every sequence, new ones included."""
    total = [_spread(case["batch"], i, case["len"], case["spread"]) for i in range(case["batch"])]
    if case["kind"] == "keep":
        return [t + case["new"] for t in total]
    return [max(t, case.get("new", 1)) for t in total]


def _news(case):
    """New tokens of every sequence."""
    return [_spread(case["batch"], i + 1, case["new"], 0.7) if case["ragged"] else case["new"]
            for i in range(case["batch"])]


def _kept(case):
    """(first place that tokens move to, number of them) of every sequence."""
    total = _totals(case)
    if case["each"]:
        return [0] * len(total), [min(t, case["kept"]) for t in total]
    return [t - case["new"] for t in total], [_spread(len(total), i + 2, case["kept"], 0.9) for i in range(len(total))]


def _offsets(counts):
    off = [0]
    for c in counts:
        off.append(off[-1] + c)
    return off


def _parents(case):
    """Trees as a drafting model's best continuations leave them: deep and with branches, parents before children. Those
    of a batch differ; they are the same for every seed (their sizes are the case's)."""
    g = torch.Generator().manual_seed(11)
    out = []
    for n in _news(case):
        p = torch.arange(n) - 1 - (torch.rand(n, generator=g) ** 2 * 4).long()
        out.append(p.clamp(min=-1))
    return torch.cat(out).to(torch.int32)


def _paths(parents, news):
    """Ancestors-or-self of every drafted token, as lists."""
    out, at = [], 0
    p = parents.tolist()
    for n in news:
        rows = []
        for i in range(n):
            rows.append((rows[p[at + i]] if p[at + i] >= 0 else []) + [i])
        out.append(rows)
        at += n
    return out


# ---------------------------------------------------------------- inputs
def _table(per, seed):
    """Page tables of sequences with `per` pages each, pages in a random order."""
    table = torch.full((len(per), max(1, max(per))), -1, dtype=torch.int32)
    order = torch.randperm(max(1, sum(per)), generator=torch.Generator().manual_seed(seed), dtype=torch.int32)
    at = 0
    for i, p in enumerate(per):
        table[i, :p] = order[at:at + p]
        at += p
    return table.cuda()


def _cache(case, g):
    """A pool of pages with codes and scales as a served model leaves them."""
    total = _totals(case)
    page, hkv, d = case["page"], case["hkv"], case["d"]
    per = [-(-t // page) for t in total]
    n = max(1, sum(per))
    s = {"pages": _table(per, 7), "lens": torch.tensor(total, dtype=torch.int32).cuda()}
    for name in ("K", "V"):
        codes = torch.empty((n, hkv, page, d), device="cuda",
                            dtype=torch.int8 if case["fmt"] == "int8" else torch.float8_e4m3fn)
        step = max(1, (1 << 28) // (hkv * page * d))
        # keys have a few channels that are larger than the others, values do not
        wide_ch = torch.exp(0.4 * torch.randn(d, generator=g, device="cuda")) if name == "K" else 1.0
        for a in range(0, n, step):
            x = torch.randn((min(step, n - a), hkv, page, d), generator=g, device="cuda") * wide_ch
            if case["fmt"] == "int8":
                codes[a:a + step] = (x * 32.0).round().clamp(-127, 127).to(torch.int8)
            else:
                codes[a:a + step] = (x * 110.0).clamp(-448, 448).to(torch.float8_e4m3fn)
        scale = torch.exp(0.3 * torch.randn((n, hkv, page // BLOCK), generator=g, device="cuda"))
        s[name] = codes
        s["k_scale" if name == "K" else "v_scale"] = scale / (32.0 if case["fmt"] == "int8" else 110.0)
    return s


def _choice(case, g):
    """Places that stay, per sequence (and head), in order; -1 behind the last."""
    total, (start, kept) = _totals(case), _kept(case)
    heads = case["hkv"] if case["each"] else 1
    idx = torch.full((case["batch"], heads, max(kept)), -1, dtype=torch.int32, device="cuda")
    for i, (t, a, k) in enumerate(zip(total, start, kept)):
        w = torch.rand((heads, t - a), generator=g, device="cuda")
        if case["each"]:
            w[:, :4] = 2.0                                      # the first tokens always stay, and the last ones
            w[:, max(0, t - k // 8):] = 2.0
        idx[i, :, :k] = (a + w.topk(k, dim=1).indices.sort(dim=1).values).to(torch.int32)
    return idx if case["each"] else idx[:, 0].contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind == "select":
        total = _totals(case)
        width = -(-max(total) // 64) * 64
        # attention sums: a few tokens get most of it, some nothing that fp32 holds, none behind the end
        w = torch.exp(2.0 * torch.randn((case["batch"], case["hkv"], width), generator=g, device="cuda"))
        w *= torch.rand(w.shape, generator=g, device="cuda") > 0.1
        s["lens"] = torch.tensor(total, dtype=torch.int32).cuda()
        w *= torch.arange(width, device="cuda") < s["lens"][:, None, None]
        s["w"], s["w_out"] = w, torch.empty_like(w)
        return s
    dtype = TYPES[case["dtype"]]
    s.update(_cache(case, g))
    if own:  # the cache handle that a program keeps (the same tensors)
        import paper_2412_09282_gb300 as P
        s["handle"] = P.KVCache(s["K"], s["V"], s["k_scale"], s["v_scale"], s["pages"], s["lens"])
    if kind == "keep":
        start, kept = _kept(case)
        s["idx"] = _choice(case, g)
        s["start"] = torch.tensor(start, dtype=torch.int32).cuda()
        s["count"] = torch.tensor(kept, dtype=torch.int32).cuda()
        first = [a // BLOCK * BLOCK for a in start]              # (the block that they join comes back whole)
        rows = [a - f + k for a, f, k in zip(start, first, kept)]
        s["from"] = torch.tensor(first, dtype=torch.int32).cuda()
        s["off"] = torch.tensor(_offsets(rows), dtype=torch.int32).cuda()
        s["n_read"], s["n_blocks"] = sum(rows), sum(-(-r // BLOCK) for r in rows)
        s["to"] = s
        if not case["in_place"]:  # other pages, which hold the tokens before the first moved one already
            to = {"lens": (s["start"] + s["count"]).to(torch.int32)}
            per = [-(-(a + k) // case["page"]) for a, k in zip(start, kept)]
            to["pages"] = _table(per, 13)
            n = max(1, sum(per))
            for name in ("K", "V"):
                to[name] = torch.zeros((n, *s[name].shape[1:]), dtype=s[name].dtype, device="cuda")
            for name in ("k_scale", "v_scale"):
                to[name] = torch.zeros((n, *s[name].shape[1:]), device="cuda")
            p = s["from"][_owner(s["off"], s["n_read"])].long()
            b = _owner(s["off"], s["n_read"])
            p = p + torch.arange(s["n_read"], device="cuda") - s["off"][b]
            old = p < s["start"][b]
            b, p = b[old], p[old]
            at, src = to["pages"][b, p // case["page"]].long(), s["pages"][b, p // case["page"]].long()
            slot = p % case["page"]
            for name, scales in (("K", "k_scale"), ("V", "v_scale")):
                to[name].view(torch.uint8)[at, :, slot] = s[name].view(torch.uint8)[src, :, slot]
                to[scales][at, :, slot // BLOCK] = s[scales][src, :, slot // BLOCK]
            s["to"] = to
        if own:
            to = s["to"]
            s["to_handle"] = s["handle"] if case["in_place"] else P.KVCache(
                to["K"], to["V"], to["k_scale"], to["v_scale"], to["pages"], to["lens"])
        return s
    new = _news(case)
    s["n_new"], s["max_new"] = sum(new), max(new)
    s["new_off"] = torch.tensor(_offsets(new), dtype=torch.int32).cuda() if case["ragged"] else None
    # (a trained model's scores are peaked: queries of more than unit size)
    s["q"] = (2.5 * torch.randn((s["n_new"], case["hq"], case["d"]), generator=g, device="cuda")).to(dtype)
    if kind == "tree":
        s["parents"] = _parents(case).cuda()
        return s
    # what attention returned beside its outputs
    lse = torch.empty((s["n_new"], case["hq"]), device="cuda")
    off, total = _offsets(new), _totals(case)
    for i, (t, c) in enumerate(zip(total, new)):
        if c:
            x, _ = _score64(s, i, t, c, off[i], torch.float32)
            lse[off[i]:off[i] + c] = torch.logsumexp(x, -1).reshape(-1, c).t()
    s["lse"] = lse
    s["w"] = None
    s["w_out"] = torch.empty((case["batch"], case["hkv"], s["pages"].shape[1] * case["page"]), device="cuda")
    if case["before"]:
        s["w"] = torch.exp(torch.randn(s["w_out"].shape, generator=g, device="cuda")) * 0.01
        s["w"] *= torch.arange(s["w"].shape[2], device="cuda") < s["lens"][:, None, None]
    return s


# ---------------------------------------------------------------- plain forms (fp32)
def _owner(off, n):
    """Sequence of each of n rows that lie one sequence after another."""
    return torch.searchsorted(off, torch.arange(n, device="cuda", dtype=off.dtype), right=True) - 1


def _new_off(s):
    c = s["case"]
    if s["new_off"] is not None:
        return s["new_off"].long()
    return torch.arange(0, s["n_new"] + 1, c["new"], device="cuda")


def _to_codes(x, fmt):
    if fmt == "int8":
        return x.round().clamp(-127.0, 127.0)
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).float()


def _rows(s):
    """Sequence and index in it of every new token, and the first new token's place."""
    noff = _new_off(s)
    b = _owner(noff, s["n_new"])
    return b, torch.arange(s["n_new"], device="cuda") - noff[b], s["lens"].long() - (noff[1:] - noff[:-1])


def _values(s, codes, scales):
    """All cached values, sequences x heads x tokens x d, 0 where there are none."""
    c = s["case"]
    t = torch.arange(c["len"], device="cuda")
    pg, slot = s["pages"][:, t // c["page"]].long().clamp(min=0), t % c["page"]
    x = codes[pg, :, slot].float() * scales[pg, :, slot // BLOCK].unsqueeze(-1)
    return torch.where((t < s["lens"][:, None])[:, :, None, None], x, 0.0).transpose(1, 2)


def _scores(s, b, j):
    """Scores, sequences x kv heads x group x new tokens x tokens."""
    c = s["case"]
    n, hkv, m, g = c["batch"], c["hkv"], s["max_new"], c["hq"] // c["hkv"]
    q = torch.zeros((n, m, c["hq"], c["d"]), device="cuda")
    q[b, j] = s["q"].float()
    q = q.view(n, m, hkv, g, c["d"]).permute(0, 2, 3, 1, 4).reshape(n, hkv, g * m, c["d"])
    x = q @ _values(s, s["K"], s["k_scale"]).transpose(2, 3)
    return x.view(n, hkv, g, m, c["len"]) * (1.0 / math.sqrt(c["d"]))


def _tree(s):
    c = s["case"]
    n, hq, hkv, d, L, m = c["batch"], c["hq"], c["hkv"], c["d"], c["len"], s["max_new"]
    b, j, held = _rows(s)
    # ancestors: powers of the parent relation, twice as far each time
    see = torch.zeros((n, m, m + 1), device="cuda")
    see[b, j, s["parents"].long() + 1] = 1.0
    see = see[:, :, 1:] + torch.eye(m, device="cuda")
    for _ in range((m - 1).bit_length()):
        see = ((see @ see) > 0).float()
    t = torch.arange(L, device="cuda")
    drafted = t - held[:, None]                                                # sequences x tokens
    seen = torch.gather(see, 2, drafted.clamp(0, m - 1)[:, None, :].expand(n, m, L)) > 0
    first = torch.zeros((n, m), device="cuda", dtype=torch.long)
    if c["window"]:
        depth = see.sum(-1).long() - 1
        first = held[:, None] + depth - c["window"] + 1
        near = depth[:, :, None] - depth[:, None, :] < c["window"]
        seen &= torch.gather(near, 2, drafted.clamp(0, m - 1)[:, None, :].expand(n, m, L))
    seen = torch.where((drafted < 0)[:, None, :], t >= first[:, :, None], seen & (drafted < m)[:, None, :])
    seen &= (t < s["lens"][:, None])[:, None, :]
    score = _scores(s, b, j).masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    p = torch.exp(score - top)
    del score
    total = p.sum(-1, keepdim=True)
    o = p.view(n, hkv, -1, L) @ _values(s, s["V"], s["v_scale"])
    o = o.view(n, hkv, -1, m, d) / torch.where(total > 0, total, 1.0)
    lse = (torch.log(total) + top).squeeze(-1)
    return {"out": o.permute(0, 3, 1, 2, 4).reshape(n, m, hq, d)[b, j].to(s["q"].dtype),
            "lse": lse.permute(0, 3, 1, 2).reshape(n, m, hq)[b, j]}


def _weights(s):
    c = s["case"]
    n, hkv, L, m = c["batch"], c["hkv"], c["len"], s["max_new"]
    b, j, held = _rows(s)
    t, at = torch.arange(L, device="cuda"), held[:, None] + torch.arange(m, device="cuda")
    seen = (t <= at[:, :, None]) & (t < s["lens"][:, None])[:, None, :]
    if c["window"]:
        seen &= t > at[:, :, None] - c["window"]
    live = torch.zeros((n, m), device="cuda", dtype=torch.bool)
    live[b, j] = True
    lse = torch.zeros((n, m, c["hq"]), device="cuda")
    lse[b, j] = s["lse"]
    lse = lse.view(n, m, hkv, -1).permute(0, 2, 3, 1).unsqueeze(-1)
    p = torch.exp(_scores(s, b, j) - lse)
    p.masked_fill_(~(seen & live[:, :, None])[:, None, None], 0.0)
    w = torch.zeros(s["w_out"].shape, device="cuda")
    w[:, :, :L] = p.sum((2, 3))
    return w if s["w"] is None else w + 0.98 * s["w"]


def _select(s):
    c = s["case"]
    w, lens = s["w"], s["lens"].long()
    n, hkv, width = w.shape
    keep = min(c["keep"], width)
    t = torch.arange(width, device="cuda")
    always = (t < c["first"]) | (t >= lens[:, None] - c["recent"])
    key = torch.where(always[:, None, :], math.inf, w)
    key = torch.where((t < lens[:, None])[:, None, :], key, -math.inf)
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices[:, :, :keep]
    count = lens.clamp(max=c["keep"])
    rank = torch.arange(keep, device="cuda")
    order = torch.where(rank < count[:, None, None], order, width).sort(-1).values
    live = order < width
    out = torch.zeros_like(w)
    out[:, :, :keep] = torch.where(live, torch.gather(w, 2, order.clamp(max=width - 1)), 0.0)
    idx = torch.full((n, hkv, c["keep"]), -1, dtype=torch.int32, device="cuda")
    idx[:, :, :keep] = torch.where(live, order, -1).to(torch.int32)
    return {"idx": idx, "count": count.to(torch.int32), "weights": out}


def _keep(s):
    c = s["case"]
    page, to = c["page"], s["to"]
    dtype = TYPES[c["dtype"]]
    off, start = s["off"].long(), s["start"].long()
    b = _owner(off, s["n_read"])
    r = torch.arange(s["n_read"], device="cuda") - off[b]
    blocks = torch.cumsum((off[1:] - off[:-1] + BLOCK - 1) // BLOCK, 0)
    blk = torch.where(b > 0, blocks[(b - 1).clamp(min=0)], 0) + r // BLOCK
    p = s["from"].long()[b] + r
    moved = p >= start[b]
    idx = s["idx"] if c["each"] else s["idx"].unsqueeze(1)
    src = idx[b, :, (p - start[b]).clamp(min=0)].long()                         # rows x heads (or one)
    src = torch.where(moved[:, None], src, p[:, None]).expand(-1, c["hkv"])
    h, bb = torch.arange(c["hkv"], device="cuda"), b[:, None]
    # what was there before the first moved token stays where it is
    pg, old_pg = s["pages"][bb, src // page].long(), to["pages"][bb, p[:, None] // page].long()
    slot = src % page
    dst, at = to["pages"][b, p // page].long(), p % page
    out = {}
    for name, scales in (("K", "k_scale"), ("V", "v_scale")):
        stay = ~moved[:, None]
        had = torch.where(stay, to[scales][old_pg, h, slot // BLOCK], s[scales][pg, h, slot // BLOCK])
        code = torch.where(stay[:, :, None], to[name][old_pg, h, slot].float(), s[name][pg, h, slot].float())
        top = torch.zeros((s["n_blocks"], BLOCK, c["hkv"]), device="cuda")
        top[blk, r % BLOCK] = had
        scale = top.amax(1)[blk]
        ratio = torch.where(scale > 0, had / torch.where(scale > 0, scale, 1.0), 0.0)
        code = _to_codes(code * ratio.unsqueeze(-1), c["fmt"])
        to[name].view(torch.uint8)[dst, :, at] = code.to(to[name].dtype).view(torch.uint8)
        to[scales][dst, :, at // BLOCK] = scale
        out[name] = (code * scale.unsqueeze(-1)).to(dtype)
    return out


def run(s):
    c = s["case"]
    kind = c["kind"]
    if not own:
        return {"tree": _tree, "weights": _weights, "select": _select, "keep": _keep}[kind](s)
    import paper_2412_09282_gb300 as P
    if kind == "tree":
        mask, positions = P.crvq_tree_mask(s["parents"], c["batch"], off=s["new_off"], lens=s["lens"],
                                           max_new=s["max_new"], window=c["window"])
        out, lse = P.crvq_cache_tree_attention(s["handle"], s["q"], mask, q_off=s["new_off"], positions=positions,
                                               window=c["window"], want_lse=True)
        return {"out": out, "lse": lse}
    if kind == "weights":
        return P.crvq_cache_weights(s["handle"], s["q"], s["lse"], q_off=s["new_off"], window=c["window"],
                                    weights=s["w"], decay=0.98, out=s["w_out"])
    if kind == "select":
        idx, count = P.crvq_cache_select(s["w"], s["lens"], c["keep"], first=c["first"], recent=c["recent"],
                                         weights_out=s["w_out"])
        return {"idx": idx, "count": count, "weights": s["w_out"]}
    P.crvq_cache_keep(s["handle"], s["idx"], s["count"], start=s["start"], out=s["to_handle"])
    K, V = P.crvq_cache_read(s["to_handle"], s["from"], s["off"], s["n_read"], dtype=TYPES[c["dtype"]])
    return {"K": K, "V": V}


def work(case):
    kind = case["kind"]
    total, hkv = _totals(case), case["hkv"]
    if kind == "select":
        n, kept = float(sum(total)) * hkv, float(sum(min(t, case["keep"]) for t in total)) * hkv
        width = -(-max(total) // 64) * 64
        return {"bytes": 4.0 * (n + kept + case["batch"] * hkv * width), "flops": n}
    wide, d = BYTES[case["dtype"]], case["d"]
    if kind == "keep":
        start, kept = _kept(case)
        rows = float(sum(kept) + sum(a % BLOCK for a in start)) * hkv
        # codes and scales in and out, places, then read back (codes and scales in, values out)
        return {"bytes": 2 * rows * (3 * d + 3 * 4 / BLOCK + d * wide) + 4.0 * sum(kept) * (hkv if case["each"] else 1),
                "flops": 6.0 * rows * d}
    hq, new = case["hq"], _news(case)
    n, keys, pairs = float(sum(new)), 0.0, 0.0
    paths = _paths(_parents(case), new) if kind == "tree" else None
    for i, (t, c) in enumerate(zip(total, new)):
        held, low = t - c, t
        for k in range(c):
            depth = len(paths[i][k]) - 1 if paths else k
            lo = max(0, held + depth - case["window"] + 1) if case["window"] else 0
            pairs += max(0, held - lo) + (depth + 1 if not case["window"] else min(depth + 1, case["window"]))
            low = min(low, lo)
        keys += t - max(0, low)
    held = (1.0 if kind == "weights" else 2.0) * hkv * keys * (d + 4.0 / BLOCK)
    if kind == "weights":
        width = -(-max(total) // case["page"]) * case["page"]
        rows = 4.0 * hkv * (case["batch"] * width + (sum(total) if case["before"] else 0))
        return {"bytes": held + n * hq * (d * wide + 4) + rows, "flops": 2.0 * pairs * hq * d}
    return {"bytes": held + n * hq * (2.0 * d * wide + 4) + 4 * n, "flops": 4.0 * pairs * hq * d}


# ---------------------------------------------------------------- 64-bit results
def _e4m3_64(x):
    """The nearest e4m3 value of a 64-bit one (ties to even, saturating): 3 bits below the leading one,
    exponents from -6."""
    a = x.abs().clamp(max=448.0)
    e = torch.floor(torch.log2(a.clamp(min=2.0 ** -40)))
    e = torch.where(torch.exp2(e + 1) <= a, e + 1, torch.where(torch.exp2(e) > a, e - 1, e))
    step = torch.exp2(e.clamp(min=-6.0) - 3.0)
    return torch.copysign((a / step).round() * step, x)


def _stored(s, name, scales, i, p):
    """Codes and their scales of the tokens p of sequence i (tokens x heads x d, x 1)."""
    page = s["case"]["page"]
    pg = s["pages"][i].long()[p // page]
    return s[name][pg, :, p % page], s[scales][pg, :, p % page // BLOCK].unsqueeze(-1)


def _score64(s, i, t, c, row, dtype=torch.float64):
    """Scores of sequence i's c queries, kv heads x group x c x t, and which are seen, causally."""
    case = s["case"]
    p = torch.arange(t, device="cuda")
    k, f = _stored(s, "K", "k_scale", i, p)
    q = s["q"][row:row + c].to(dtype).view(c, case["hkv"], -1, case["d"]).permute(1, 2, 0, 3)
    x = (q @ (k.to(dtype) * f.to(dtype)).permute(1, 2, 0).unsqueeze(1)) / math.sqrt(case["d"])
    at = torch.arange(t - c, t, device="cuda")
    seen = p <= at[:, None]
    if case["window"]:
        seen &= p > at[:, None] - case["window"]
    return x.masked_fill(~seen, -math.inf), seen


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    total = _totals(case)
    if kind == "select":
        out = torch.zeros(s["w"].shape, dtype=torch.float64, device="cuda")
        for i, t in enumerate(total):
            if t <= case["keep"]:
                out[i, :, :t] = s["w"][i, :, :t].double()
                continue
            for h in range(case["hkv"]):
                w = s["w"][i, h, :t].double()
                mid = torch.arange(case["first"], t - case["recent"], device="cuda")
                left = case["keep"] - case["first"] - case["recent"]
                best = mid[torch.argsort(-w[mid], stable=True)[:left]]
                stay = torch.cat([torch.arange(case["first"], device="cuda"), best.sort().values,
                                  torch.arange(t - case["recent"], t, device="cuda")])
                out[i, h, :stay.numel()] = w[stay]
        return {"idx": None, "count": None, "weights": out}
    if kind == "keep":
        start, kept = _kept(case)
        top = (lambda x: x.round().clamp(-127, 127)) if case["fmt"] == "int8" else _e4m3_64
        out = {"K": [], "V": []}
        for i, (a, k) in enumerate(zip(start, kept)):
            f = a // BLOCK * BLOCK
            for name, scales in (("K", "k_scale"), ("V", "v_scale")):
                old, of = _stored(s, name, scales, i, torch.arange(f, a, device="cuda"))
                x, xf = [], []
                for h in range(case["hkv"]):
                    p = s["idx"][i, h if case["each"] else slice(None)][:k].long()
                    code, fac = _stored(s, name, scales, i, p)
                    x.append(torch.cat([old[:, h].double(), code[:, h].double()]))
                    xf.append(torch.cat([of[:, h].double(), fac[:, h].double()]))
                x, xf = torch.stack(x, 1), torch.stack(xf, 1)
                for r in range(0, x.shape[0], BLOCK * 512):
                    y, yf = x[r:r + BLOCK * 512], xf[r:r + BLOCK * 512]
                    n = y.shape[0]
                    pad = torch.zeros((-n % BLOCK, *yf.shape[1:]), dtype=yf.dtype, device="cuda")
                    most = torch.cat([yf, pad]).view(-1, BLOCK, *yf.shape[1:]).amax(1).repeat_interleave(BLOCK, 0)[:n]
                    out[name].append(torch.where(most > 0, top(y * (yf / most)) * most, 0.0))
        return {k: torch.cat(v) for k, v in out.items()}
    new, hkv = _news(case), case["hkv"]
    if 4.0 * sum(t * c for t, c in zip(total, new)) * case["hq"] * case["d"] > 3e12:
        return None
    off = _offsets(new)
    if kind == "weights":
        w = torch.zeros(s["w_out"].shape, dtype=torch.float64, device="cuda")
        for i, (t, c) in enumerate(zip(total, new)):
            x, _ = _score64(s, i, t, c, off[i])
            lse = s["lse"][off[i]:off[i] + c].double().view(c, hkv, -1).permute(1, 2, 0).unsqueeze(-1)
            w[i, :, :t] = torch.exp(x - lse).sum((1, 2))
        return w if s["w"] is None else w + 0.98 * s["w"].double()
    paths, out, lses = _paths(_parents(case), new), [], []
    for i, (t, c) in enumerate(zip(total, new)):
        held = t - c
        p = torch.arange(t, device="cuda")
        seen = torch.zeros((c, t), dtype=torch.bool)
        for k, path in enumerate(paths[i]):
            lo = max(0, held + len(path) - case["window"]) if case["window"] else 0
            seen[k, lo:max(held, lo)] = True
            seen[k, [held + a for a in (path[-case["window"]:] if case["window"] else path)]] = True
        seen = seen.cuda()
        k, f = _stored(s, "K", "k_scale", i, p)
        v, vf = _stored(s, "V", "v_scale", i, p)
        q = s["q"][off[i]:off[i] + c].double().view(c, hkv, -1, case["d"])
        o = torch.empty_like(q)
        lse = torch.empty((c, hkv, q.shape[2]), dtype=torch.float64, device="cuda")
        for h in range(hkv):
            kk, vv = k[:, h].double() * f[:, h].double(), v[:, h].double() * vf[:, h].double()
            x = (torch.einsum("cgd,td->cgt", q[:, h], kk) / math.sqrt(case["d"])).masked_fill(~seen[:, None], -math.inf)
            lse[:, h] = torch.logsumexp(x, -1)
            o[:, h] = torch.einsum("cgt,td->cgd", torch.softmax(x, -1), vv)
        out.append(o.reshape(c, case["hq"], case["d"]))
        lses.append(lse.reshape(c, case["hq"]))
    return {"out": torch.cat(out), "lse": torch.cat(lses)}
