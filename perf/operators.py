"""The operators of a decode step with compressed weights and cache, as cases to be timed.

- append: keys and values of new tokens, rotated by their position, into a paged cache that holds 8-bit
  codes with one scale per 16 tokens and head; the touched blocks are then read back as values.
- attend: attention of the newest tokens of every sequence over such a cache.
- q4: Y = X W^T with 4-bit weights and a scale per group of inputs.
- quantize: a weight matrix to 4-bit codes, scales and the values they stand for.

Head counts and sizes are those of the repository's workloads (4096 and 8192 channels in heads of 128,
the matrices 512 x 512, 4096 x 4096, 11008 x 4096 and 28672 x 8192, 4096 tokens) and generic ones
around them.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 16                                   # tokens per scale
TOP = {"int8": 127.0, "e4m3": 448.0}         # largest code
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # One sequence decodes one token: the smallest append, all latency.
        dict(name="append_step", kind="append", batch=1, held=1000, spread=0.0, new=1, ragged=False, page=64,
             hq=64, hkv=8, d=128, fmt="int8", dtype="bf16", style="half"),
        # Three prompts of odd lengths (4096 tokens at most) arrive at caches that end inside a block,
        # 32 heads, in the type that the products from codes return.
        dict(name="append_prompts", kind="append", batch=3, held=777, spread=0.9, new=4091, ragged=True, page=16,
             hq=32, hkv=32, d=128, fmt="e4m3", dtype="f32", style="pairs"),
        # One sequence, one token, a short cache: latency.
        dict(name="attend_step", kind="attend", batch=1, len=1001, spread=0.0, new=1, ragged=False, page=64,
             hq=64, hkv=8, d=128, fmt="int8", dtype="bf16", window=0, empty=False),
        # A serving batch of 64 sequences of very different lengths (one just started: empty), a kv head
        # per query head, the e4m3 cache.
        dict(name="attend_batch", kind="attend", batch=64, len=4096, spread=0.95, new=1, ragged=False, page=16,
             hq=32, hkv=32, d=128, fmt="e4m3", dtype="f16", window=0, empty=True),
        # Four long documents, one token each: the largest read of the cache.
        dict(name="attend_long", kind="attend", batch=4, len=131072, spread=0.2, new=1, ragged=False, page=256,
             hq=64, hkv=8, d=128, fmt="int8", dtype="bf16", window=0, empty=False),
        # Up to five drafted tokens per sequence to verify, heads of 64, fp32, a sliding window.
        dict(name="attend_draft", kind="attend", batch=16, len=3001, spread=0.7, new=5, ragged=True, page=32,
             hq=32, hkv=4, d=64, fmt="int8", dtype="f32", window=2000, empty=False),
        # Chunks of two prompts, 1024 tokens at most, over up to 8192 tokens of cache.
        dict(name="attend_chunk", kind="attend", batch=2, len=8192, spread=0.4, new=1024, ragged=True, page=64,
             hq=64, hkv=8, d=128, fmt="int8", dtype="bf16", window=0, empty=False),
        # The 512 x 512 layer, one token, fp32: the smallest product.
        dict(name="q4_512", kind="q4", M=512, N=512, b=1, group=64, zeros=False, dtype="f32"),
        # gate_proj of a 7B block, one token.
        dict(name="q4_gate", kind="q4", M=11008, N=4096, b=1, group=128, zeros=False, dtype="bf16"),
        # The 28672 x 8192 up_proj, sixteen sequences, zero points.
        dict(name="q4_up_b16", kind="q4", M=28672, N=8192, b=16, group=128, zeros=True, dtype="f16"),
        # Quantizing the small layer, and a q_proj with zero points.
        dict(name="quantize_512", kind="quantize", M=512, N=512, group=64, zeros=False, dtype="f32"),
        dict(name="quantize_q_proj", kind="quantize", M=4096, N=4096, group=128, zeros=True, dtype="f32"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choice(["append", "append", "attend", "attend", "attend", "q4", "q4", "quantize"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if kind in ("append", "attend"):
        hkv = rng.choice([1, 2, 4, 8, 32])
        hq = hkv * rng.choice([1, 1, 2, 4, 8] if hkv < 32 else [1, 2])
        c = dict(kind=kind, page=rng.choice([16, 32, 48, 64, 128, 256]), hq=hq, hkv=hkv, d=rng.choice([64, 128]),
                 fmt=rng.choice(["int8", "e4m3"]), dtype=dtype, spread=rng.choice([0.0, 0.5, 0.95]),
                 ragged=rng.random() < 0.5)
        if kind == "append":
            c["batch"] = _log(rng, 1, 64)
            c["held"] = rng.choice([0, _log(rng, 1, 8192)])
            c["new"] = rng.choice([1, 1, rng.randint(2, 8), _log(rng, 9, 4096)])
            most = 12000 * 32 * 128 // (hkv * c["d"])          # tokens of all sequences together
            c["new"] = max(1, min(c["new"], most // c["batch"]))
            c["style"] = rng.choice(["half", "pairs"])
            return c
        c["batch"] = _log(rng, 1, 64)
        c["new"] = rng.choice([1, 1, 1, rng.randint(2, 8), _log(rng, 9, 1024)])
        most = 4 * 131072 * 8 * 128 // (hkv * c["d"] * c["batch"])
        c["len"] = _log(rng, min(most, 64), min(most, 131072))
        # no more score entries than the listed chunks have
        c["new"] = max(1, min(c["new"], 2 * 64 * 1024 * 8192 // (c["batch"] * hq * c["len"])))
        c["window"] = rng.choice([0, 0, 0, _log(rng, 16, 4096)])
        c["empty"] = c["batch"] > 1 and rng.random() < 0.3
        return c
    group = rng.choice([32, 64, 128])
    zeros = rng.random() < 0.5
    if kind == "q4":
        M, N = _log(rng, 16, 28672), _log(rng, 64, 28672)
        while M * N > 28672 * 8192:
            M //= 2
        return dict(kind=kind, M=M, N=N, b=_log(rng, 1, 32), group=group, zeros=zeros, dtype=dtype)
    return dict(kind=kind, M=_log(rng, 16, 4096), N=_log(rng, 64, 4096), group=group, zeros=zeros, dtype=dtype)


# ---------------------------------------------------------------- sizes
def _spread(n, i, most, by):
    return max(1, round(most * (1.0 - by * ((i * 0.6180339887498949) % 1.0)))) if n else 0


def _sizes(case):
    """(tokens held before, new tokens) of every sequence."""
    n = case["batch"]
    new = [_spread(n, i + 1, case["new"], 0.7) if case["ragged"] else case["new"] for i in range(n)]
    if case["kind"] == "append":
        held = [_spread(n, i, case["held"], case["spread"]) if case["held"] else 0 for i in range(n)]
        return held, new
    total = [_spread(n, i, case["len"], case["spread"]) for i in range(n)]
    if case["empty"]:
        total[-1] = 0
    return [max(0, t - c) for t, c in zip(total, new)], new


def _totals(case):
    held, new = _sizes(case)
    if case["kind"] == "append":
        return [h + c for h, c in zip(held, new)]
    total = [_spread(case["batch"], i, case["len"], case["spread"]) for i in range(case["batch"])]
    if case["empty"]:
        total[-1] = 0
    return total


def _read_sizes(case):
    """First token and number of tokens of every sequence's touched blocks."""
    held, new = _sizes(case)
    start = [h // BLOCK * BLOCK for h in held]
    return start, [h + c - s for h, c, s in zip(held, new, start)]


def _offsets(counts):
    off = [0]
    for c in counts:
        off.append(off[-1] + c)
    return off


# ---------------------------------------------------------------- inputs
def _cache(case, g):
    """A pool of pages in a random order with codes and scales as a served model leaves them."""
    total = _totals(case)
    page, hkv, d = case["page"], case["hkv"], case["d"]
    per = [-(-t // page) for t in total]
    wide = max(1, max(per))
    n = max(1, sum(per))
    table = torch.full((case["batch"], wide), -1, dtype=torch.int32)
    order = torch.randperm(n, generator=torch.Generator().manual_seed(7), dtype=torch.int32)
    at = 0
    for i, p in enumerate(per):
        table[i, :p] = order[at:at + p]
        at += p
    s = {"pages": table.cuda(), "lens": torch.tensor(total, dtype=torch.int32).cuda()}
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


def _q4_weights(case, g):
    M, N, group = case["M"], case["N"], case["group"]
    row = -(-((N + 1) // 2) // 16) * 16                        # rows on 16-byte boundaries
    codes = torch.randint(0, 256, (M, row), generator=g, device="cuda", dtype=torch.uint8)
    G = -(-N // group)
    scales = (0.004 * torch.exp(0.3 * torch.randn((M, G), generator=g, device="cuda"))).to(torch.bfloat16)
    zeros = torch.randint(4, 12, (M, G), generator=g, device="cuda", dtype=torch.uint8) if case["zeros"] else None
    return codes[:, :(N + 1) // 2], scales, zeros


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, dtype = case["kind"], TYPES[case["dtype"]]
    s = {"case": case}
    if kind == "quantize":
        W = 0.02 * torch.randn((case["M"], case["N"]), generator=g, device="cuda")
        W[:, :max(1, case["N"] // 100)] *= 10.0
        s["W"] = W.to(dtype)
        return s
    if kind == "q4":
        s["codes"], s["scales"], s["zeros"] = _q4_weights(case, g)
        wide_ch = torch.exp(0.5 * torch.randn(case["N"], generator=g, device="cuda"))
        s["X"] = (torch.randn((case["b"], case["N"]), generator=g, device="cuda") * wide_ch).to(dtype)
        if own:  # the handle that a program makes once around its weights (no other layout)
            import paper_2412_09282_gb300 as P
            s["handle"] = P.Q4Matrix(s["codes"], s["scales"], s["zeros"], case["N"], case["group"])
        return s
    s.update(_cache(case, g))
    held, new = _sizes(case)
    s["n_new"] = sum(new)
    s["new_off"] = torch.tensor(_offsets(new), dtype=torch.int32).cuda() if case["ragged"] else None
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if kind == "append":
        # one fused projection's output: q, k and v are views of its rows
        qkv = torch.randn((s["n_new"], hq + 2 * hkv, d), generator=g, device="cuda").to(dtype)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        ang = torch.outer(torch.arange(max(_totals(case)), dtype=torch.float64),
                          10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d))
        s["cos"], s["sin"] = ang.cos().float().cuda(), ang.sin().float().cuda()
        start, count = _read_sizes(case)
        s["start"] = torch.tensor(start, dtype=torch.int32).cuda()
        s["off"] = torch.tensor(_offsets(count), dtype=torch.int32).cuda()
        s["n_read"], s["n_blocks"] = sum(count), sum(-(-c // BLOCK) for c in count)
    else:
        # (a trained model's scores are peaked: queries of more than unit size)
        s["q"] = (2.5 * torch.randn((s["n_new"], hq, d), generator=g, device="cuda")).to(dtype)
        s["max_new"] = max(new)
    if own:  # the cache handle that a program keeps (the same tensors)
        import paper_2412_09282_gb300 as P
        s["handle"] = P.KVCache(s["K"], s["V"], s["k_scale"], s["v_scale"], s["pages"], s["lens"])
    return s


# ---------------------------------------------------------------- plain forms (fp32)
def _owner(off, n):
    """Sequence of each of n rows that lie one sequence after another."""
    return torch.searchsorted(off, torch.arange(n, device="cuda", dtype=off.dtype), right=True) - 1


def _new_off(s):
    c = s["case"]
    if s["new_off"] is not None:
        return s["new_off"]
    return torch.arange(0, s["n_new"] + 1, c["new"], device="cuda", dtype=torch.int32)


def _rotate(x, cos, sin, style):
    x, cos, sin = x.float(), cos.unsqueeze(1), sin.unsqueeze(1)
    if style == "half":
        a, b = x.chunk(2, dim=-1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)


def _to_codes(x, fmt):
    if fmt == "int8":
        return x.round().clamp(-127.0, 127.0)
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).float()


def _append(s):
    c = s["case"]
    page = c["page"]
    noff, lens, off = _new_off(s), s["lens"].long(), s["off"].long()
    count = (noff[1:] - noff[:-1]).long()
    held = lens - count
    b = _owner(noff, s["n_new"])
    pos = held[b] + torch.arange(s["n_new"], device="cuda") - noff[b]
    cos, sin = s["cos"][pos], s["sin"][pos]
    fresh = {"K": _rotate(s["k"], cos, sin, c["style"]), "V": s["v"].float()}
    # the touched blocks' tokens, in rows: block, slot in it, place in the cache, index among the new ones
    b = _owner(off, s["n_read"])
    r = torch.arange(s["n_read"], device="cuda") - off[b]
    blocks = torch.cumsum((off[1:] - off[:-1] + BLOCK - 1) // BLOCK, 0)
    blk = torch.where(b > 0, blocks[(b - 1).clamp(min=0)], 0) + r // BLOCK
    pos = s["start"][b] + r
    pg, slot = s["pages"][b, pos // page].long(), pos % page
    new = pos >= held[b]
    at = (noff[b] + pos - held[b]).clamp(min=0)
    out = {"q": _rotate(s["q"], cos, sin, c["style"]).to(s["q"].dtype)}
    for name, scales in (("K", s["k_scale"]), ("V", s["v_scale"])):
        x = torch.where(new[:, None, None], fresh[name][at], 0.0)
        had = scales[pg, :, slot // BLOCK]                                     # rows x heads
        old = torch.where(new[:, None, None], 0.0, s[name][pg, :, slot].float())
        top = torch.zeros((s["n_blocks"], BLOCK, c["hkv"]), device="cuda")
        top[blk, r % BLOCK] = x.abs().amax(-1)
        kept = torch.zeros((s["n_blocks"], BLOCK, c["hkv"]), device="cuda")
        kept[blk, r % BLOCK] = torch.where(new[:, None], 0.0, had)
        scale = torch.maximum(kept.amax(1), top.amax(1) * (1.0 / TOP[c["fmt"]]))[blk]
        safe = torch.where(scale > 0, scale, 1.0).unsqueeze(-1)
        code = torch.where(new[:, None, None], _to_codes(x / safe, c["fmt"]),
                           _to_codes(old * (had.unsqueeze(-1) / safe), c["fmt"]))
        out[name] = code * scale.unsqueeze(-1)
    return out


def _attend(s):
    c = s["case"]
    n, hq, hkv, d = c["batch"], c["hq"], c["hkv"], c["d"]
    L, m, g = c["len"], s["max_new"], c["hq"] // c["hkv"]
    noff, lens = _new_off(s).long(), s["lens"].long()
    count = noff[1:] - noff[:-1]
    b = _owner(noff, s["n_new"])
    j = torch.arange(s["n_new"], device="cuda") - noff[b]
    t = torch.arange(L, device="cuda")
    pg, slot = s["pages"][:, t // c["page"]].long().clamp(min=0), t % c["page"]
    held = t < lens[:, None]                                                   # sequences x tokens

    def values(codes, scales):
        x = codes[pg, :, slot].float() * scales[pg, :, slot // BLOCK].unsqueeze(-1)
        return torch.where(held[:, :, None, None], x, 0.0).transpose(1, 2)     # sequences x heads x tokens x d

    q = torch.zeros((n, m, hq, d), device="cuda")
    q[b, j] = s["q"].float()
    q = q.view(n, m, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, g * m, d)
    score = (q @ values(s["K"], s["k_scale"]).transpose(2, 3)).view(n, hkv, g, m, L) * (1.0 / math.sqrt(d))
    at = (lens - count)[:, None] + torch.arange(m, device="cuda")              # position of every query
    seen = held[:, None, :] & (t <= at[:, :, None])
    if c["window"]:
        seen = seen & (t > at[:, :, None] - c["window"])
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top > -math.inf, top, 0.0))
    del score
    total = p.sum(-1, keepdim=True)
    o = p.view(n, hkv, g * m, L) @ values(s["V"], s["v_scale"])
    o = o.view(n, hkv, g, m, d) / torch.where(total > 0, total, 1.0)
    return o.permute(0, 3, 1, 2, 4).reshape(n, m, hq, d)[b, j].to(s["q"].dtype)


def _q4(s):
    c = s["case"]
    codes = s["codes"]
    q = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(1)[:, :c["N"]].float()
    grp = torch.arange(c["N"], device="cuda") // c["group"]
    z = 8.0 if s["zeros"] is None else s["zeros"].float()[:, grp]
    return (s["X"].float() @ ((q - z) * s["scales"].float()[:, grp]).t()).to(s["X"].dtype)


def _quantize(s):
    c = s["case"]
    M, N, group = c["M"], c["N"], c["group"]
    G = -(-N // group)
    W = torch.zeros((M, G * group), device="cuda")
    W[:, :N] = s["W"].float()
    W = W.view(M, G, group)
    if c["zeros"]:
        lo = W.amin(2).clamp(max=0.0)
        scale = ((W.amax(2).clamp(min=0.0) - lo) * (1.0 / 15.0)).to(torch.bfloat16)
        f = scale.float()
        safe = torch.where(f > 0, f, 1.0)
        z = (-lo / safe).round().clamp(0.0, 15.0)
    else:
        scale = (W.abs().amax(2) * (1.0 / 7.0)).to(torch.bfloat16)
        f = scale.float()
        safe = torch.where(f > 0, f, 1.0)
        z = torch.full_like(f, 8.0)
    q = ((W / safe.unsqueeze(2)).round() + z.unsqueeze(2)).clamp(0.0, 15.0)
    W_hat = ((q - z.unsqueeze(2)) * f.unsqueeze(2)).view(M, -1)[:, :N]
    return {"W_hat": W_hat, "scales": scale}


def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"append": _append, "attend": _attend, "q4": _q4, "quantize": _quantize}[kind](s)
    import paper_2412_09282_gb300 as P
    c = s["case"]
    if kind == "append":
        q = P.crvq_cache_append(s["handle"], s["k"], s["v"], new_off=s["new_off"], cos=s["cos"], sin=s["sin"],
                                interleaved=c["style"] == "pairs", q=s["q"])
        K, V = P.crvq_cache_read(s["handle"], s["start"], s["off"], s["n_read"])
        return {"q": q, "K": K, "V": V}
    if kind == "attend":
        return P.crvq_cache_attention(s["handle"], s["q"], q_off=s["new_off"], window=c["window"])
    if kind == "q4":
        return P.crvq_q4_matvec(s["X"], s["handle"])
    m, W_hat = P.crvq_q4_quantize(s["W"], c["group"], symmetric=not c["zeros"], want_W_hat=True)
    return {"W_hat": W_hat, "scales": m.scales}


def work(case):
    kind, wide = case["kind"], BYTES[case["dtype"]]
    if kind in ("q4", "quantize"):
        M, N = float(case["M"]), float(case["N"])
        held = M * N / 2 + M * math.ceil(N / case["group"]) * (3 if case["zeros"] else 2)
        if kind == "q4":
            return {"bytes": held + case["b"] * (M + N) * wide, "flops": 2.0 * case["b"] * M * N}
        return {"bytes": held + M * N * (wide + 4), "flops": 6.0 * M * N}
    held, new = _sizes(case)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    n = float(sum(new))
    if kind == "append":
        start, count = _read_sizes(case)
        rows, old = float(sum(count)), float(sum(h - a for h, a in zip(held, start)))
        scales = 8.0 * hkv * sum(-(-c // BLOCK) for c in count)
        # new k, v, q in; rotated q out; old codes of the touched blocks in, all their codes and scales
        # out; then read back (codes and scales in, fp32 values out)
        return {"bytes": n * d * wide * (2 * hq + 2 * hkv) + n * d * 4 + 2.0 * d * hkv * (old + 2 * rows)
                + 3 * scales + 8.0 * rows * hkv * d,
                "flops": 3.0 * n * d * (hq + hkv) + 4.0 * rows * hkv * d}
    keys = pairs = 0.0
    for t, c in zip(_totals(case), new):
        first = max(0, t - c - case["window"] + 1) if case["window"] else 0
        keys += t - min(first, t)
        for k in (range(c) if c <= 64 else range(0, c, 16)):
            at = t - c + k
            lo = max(0, at - case["window"] + 1) if case["window"] else 0
            pairs += max(0, at + 1 - lo) * (1 if c <= 64 else min(16, c - k))
    return {"bytes": 2.0 * keys * hkv * d + 8.0 * hkv * keys / BLOCK + 2.0 * n * hq * d * wide,
            "flops": 4.0 * pairs * hq * d}


# ---------------------------------------------------------------- 64-bit results
def _e4m3_64(x):
    """The nearest e4m3 value of a 64-bit one (ties to even, saturating): 3 bits below the leading one,
    exponents from -6."""
    a = x.abs().clamp(max=448.0)
    e = torch.floor(torch.log2(a.clamp(min=2.0 ** -40)))
    e = torch.where(torch.exp2(e + 1) <= a, e + 1, torch.where(torch.exp2(e) > a, e - 1, e))
    step = torch.exp2(e.clamp(min=-6.0) - 3.0)
    return torch.copysign((a / step).round() * step, x)


def _turn64(x, cos, sin, style):
    y = torch.empty_like(x)
    h = x.shape[-1] // 2
    first, second = (slice(0, h), slice(h, None)) if style == "half" else (slice(0, None, 2), slice(1, None, 2))
    y[..., first] = x[..., first] * cos - x[..., second] * sin
    y[..., second] = x[..., first] * sin + x[..., second] * cos
    return y


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "quantize":
        W = s["W"].double()
        M, N = W.shape
        W_hat, scales = torch.empty_like(W), []
        for a in range(0, N, case["group"]):
            w = W[:, a:a + case["group"]]
            if case["zeros"]:
                lo = w.min(1, keepdim=True).values.clamp(max=0.0)
                f = ((w.max(1, keepdim=True).values.clamp(min=0.0) - lo) / 15.0).to(torch.bfloat16)
                d = torch.where(f > 0, f.double(), 1.0)
                z = torch.round(-lo / d).clamp(0, 15)
            else:
                f = (w.abs().max(1, keepdim=True).values / 7.0).to(torch.bfloat16)
                d, z = torch.where(f > 0, f.double(), 1.0), 8.0
            k = (torch.round(w / d) + z).clamp(0, 15)
            W_hat[:, a:a + case["group"]] = (k - z) * f.double()
            scales.append(f.double())
        return {"W_hat": W_hat, "scales": torch.cat(scales, 1)}
    if kind == "q4":
        X = s["X"].double()
        Y = torch.zeros((case["b"], case["M"]), dtype=torch.float64, device="cuda")
        for k, a in enumerate(range(0, case["N"], case["group"])):
            e = min(case["N"], a + case["group"])
            byte = s["codes"][:, a // 2:(e + 1) // 2].long()
            v = torch.empty((case["M"], 2 * byte.shape[1]), dtype=torch.float64, device="cuda")
            v[:, 0::2], v[:, 1::2] = (byte % 16).double(), (byte // 16).double()
            z = 8.0 if s["zeros"] is None else s["zeros"][:, k:k + 1].double()
            Y += (X[:, a:e] @ (v[:, :e - a] - z).t()) * s["scales"][:, k].double()
        return Y
    held, new = _sizes(case)
    noff, page = _offsets(new), case["page"]
    table = s["pages"].tolist()

    def stored(name, scales, i, first, last):
        """Codes and their scales of the tokens [first, last) of sequence i (tokens x heads x d, x 1)."""
        p = torch.arange(first, last, device="cuda")
        pg = torch.tensor(table[i], device="cuda")[p // page]
        return s[name][pg, :, p % page].double(), s[scales][pg, :, p % page // BLOCK].double().unsqueeze(-1)

    if kind == "append":
        out = {"q": [], "K": [], "V": []}
        top = TOP[case["fmt"]]
        to_code = (lambda x: x.round().clamp(-127, 127)) if case["fmt"] == "int8" else _e4m3_64
        for i, (h, c) in enumerate(zip(held, new)):
            cos, sin = (s[k][h:h + c].double().unsqueeze(1) for k in ("cos", "sin"))
            rows = slice(noff[i], noff[i] + c)
            out["q"].append(_turn64(s["q"][rows].double(), cos, sin, case["style"]))
            fresh = {"K": _turn64(s["k"][rows].double(), cos, sin, case["style"]), "V": s["v"][rows].double()}
            for name, scales in (("K", "k_scale"), ("V", "v_scale")):
                for a in range(h // BLOCK * BLOCK, h + c, BLOCK):
                    x = fresh[name][max(0, a - h):a + BLOCK - h]
                    f = x.abs().amax((0, 2)).view(1, -1, 1) / top
                    parts = []
                    if a < h:
                        old, had = stored(name, scales, i, a, h)
                        f = torch.maximum(f, had[:1])
                        parts.append(to_code(old * had / f) * f)
                    parts.append(torch.where(f > 0, to_code(x / f) * f, 0.0))
                    out[name] += parts
        return {k: torch.cat(v) for k, v in out.items()}
    total, hkv = _totals(case), case["hkv"]
    if 4.0 * sum(t * c for t, c in zip(total, new)) * case["hq"] * case["d"] > 3e12:
        return None
    out = []
    for i, (t, c) in enumerate(zip(total, new)):
        q = s["q"][noff[i]:noff[i] + c].double().view(c, hkv, -1, case["d"])
        o = torch.zeros_like(q)
        at = torch.arange(t - c, t, device="cuda")
        pos = torch.arange(t, device="cuda")
        seen = pos <= at[:, None]
        if case["window"]:
            seen &= pos > at[:, None] - case["window"]
        live = seen.any(1)
        if bool(live.any()):
            K, ks = stored("K", "k_scale", i, 0, t)
            V, vs = stored("V", "v_scale", i, 0, t)
            for h in range(hkv):
                k, v = K[:, h] * ks[:, h], V[:, h] * vs[:, h]
                z = torch.einsum("cgd,td->gct", q[:, h], k) / math.sqrt(case["d"])
                w = torch.softmax(z.masked_fill(~seen, -math.inf)[:, live], dim=-1)
                o[live, h] = torch.einsum("gct,td->cgd", w, v)
        out.append(o.reshape(c, case["hq"], case["d"]))
    return torch.cat(out)
