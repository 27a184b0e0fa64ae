"""Caches and inputs for the decode-step tests: small paged caches with hostile contents wherever no
token lies (NaN codes and NaN scales), on the host for the oracle and on the GPU for the calls."""
import numpy as np
import torch

from oracle import decode_oracle as D

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# unit roundoff of an output, and of a softmax weight as the kernel holds it
OUT_ROUND = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}   # 24, 8 and 11 significant bits
WEIGHT_ROUND = {"f32": 2.0 ** -21, "bf16": 2.0 ** -11, "f16": 2.0 ** -11}


def make(seed, lens, page, n_kv, d, fmt, spare=2, wide=None, page_gap=0):
    """(oracle cache dict, P.KVCache): lens tokens per sequence with random codes and scales."""
    rng = np.random.default_rng(seed)
    per = [-(-n // page) for n in lens]
    n_pages = sum(per) + spare
    order = rng.permutation(n_pages).astype(np.int32)
    wide = wide or max(1, max(per))
    pages = np.full((len(lens), wide), -7, np.int32)          # entries past the end are never looked up
    at = 0
    for b, n in enumerate(per):
        pages[b, :n] = order[at:at + n]
        at += n
    host = {"pages": pages, "lens": np.asarray(lens, np.int32)}
    garbage = np.float32(-128.0 if fmt == "int8" else np.nan)
    for name, scales in (("K", "k_scale"), ("V", "v_scale")):
        c = np.full((n_pages, n_kv, page, d), garbage, np.float32)
        s = np.full((n_pages, n_kv, page // 16), np.nan, np.float32)
        for b, n in enumerate(lens):
            for p in range(n):
                pg, i = D.place(pages, page, b, p)
                x = rng.standard_normal((n_kv, d)).astype(np.float32) * (40 if fmt == "int8" else 120)
                c[pg, :, i] = D.to_codes(x, fmt)
                if i % 16 == 0:
                    s[pg, :, i // 16] = np.exp(0.5 * rng.standard_normal(n_kv)) / (40 if fmt == "int8" else 120)
        host[name], host[scales] = c, s
    return host, on_gpu(host, fmt, page_gap)


def on_gpu(host, fmt, page_gap=0):
    """P.KVCache with the host cache's contents; page_gap: unused 16-byte rows between pages."""
    import paper_2412_09282_gb300 as P
    dt = torch.int8 if fmt == "int8" else torch.float8_e4m3fn
    t = {}
    for name in ("K", "V"):
        x = torch.from_numpy(host[name])
        codes = x.to(torch.int8) if fmt == "int8" else x.to(torch.float8_e4m3fn)
        n, h, p, d = codes.shape
        pool = torch.zeros((n, h * p * d + 16 * page_gap), dtype=torch.uint8)
        pool[:, :h * p * d] = codes.contiguous().view(torch.uint8).view(n, -1)
        pool = pool.cuda()
        t[name] = pool.view(dt).as_strided((n, h, p, d), (pool.stride(0), p * d, d, 1))
    return P.KVCache(t["K"], t["V"], *(torch.from_numpy(host[k].copy()).cuda()
                                       for k in ("k_scale", "v_scale", "pages", "lens")))


def offsets(counts):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32).cuda()


def heads(x, dtype, gap=0):
    """A tokens x heads x d tensor of `dtype` as a view with gap unused elements after each row."""
    t = torch.from_numpy(np.ascontiguousarray(x)).to(TORCH[dtype]).cuda()
    if not gap:
        return t
    n, h, d = t.shape
    buf = torch.zeros(n * (h * d + gap) + 8, dtype=t.dtype, device="cuda")[1 if gap % 2 else 0:]
    v = buf.as_strided((n, h, d), (h * d + gap, d, 1))
    v.copy_(t)
    return v


def exactly(t):
    """The host fp32 values of a device tensor."""
    return t.detach().float().cpu().numpy()
