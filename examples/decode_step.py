"""Serving one attention layer from compressed memory: three prompts, then tokens one by one.

The layer's query, key and value projections are 4-bit (crvq_q4_quantize, crvq_q4_matvec), its keys and
values are cached in 8 bits (crvq_cache_append, crvq_cache_attention), and its output projection is the
vector-quantized 512 x 512 layer, multiplied straight from its codes (crvq_lut_matvec). A token's step is
captured once in a CUDA graph and replayed: the lengths that every call depends on are on the device.

    python examples/decode_step.py [--tokens 64] [--format int8|e4m3]

Prints the time of a step and how far the last step's attention is from the same in fp64 over the values
that the cache holds (crvq_cache_read).
"""
import argparse
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2412_09282_gb300 as P
import synthetic as S

HEADS, KV_HEADS, HEAD_DIM, PAGE = 8, 2, 64, 64
WIDTH = HEADS * HEAD_DIM


class Layer:
    """Weights, cache and rotation tables of one layer for a fixed set of sequences."""

    def __init__(self, n_seq, longest, fmt, seed=0):
        g = torch.Generator().manual_seed(seed)
        cfg = S.C1
        W_qkv = 0.05 * torch.randn((WIDTH + 2 * KV_HEADS * HEAD_DIM, WIDTH), generator=g)
        self.qkv, _ = P.crvq_q4_quantize(W_qkv.cuda(), group=64)
        W_o, X = torch.from_numpy(S.gen_W(cfg)).cuda(), torch.from_numpy(S.gen_X(cfg)).cuda()
        out = P.crvq_quantize_layer(W_o, X, cfg)
        covered = out.report["n_crit_groups"]
        self.perm = out.perm
        self.books = [P.Codebook(out.C_base, out.codes_base, cfg.N // 8)] + [
            P.Codebook(out.C_ext[t].contiguous(), out.codes_ext[t], covered) for t in range(cfg.n_ext)]
        angle = torch.arange(longest)[:, None] / 10000.0 ** (torch.arange(HEAD_DIM // 2) / (HEAD_DIM / 2))
        self.cos, self.sin = angle.cos().float().cuda(), angle.sin().float().cuda()
        per = -(-longest // PAGE)
        pages = torch.randperm(n_seq * per, generator=g, dtype=torch.int32).view(n_seq, per)
        self.lens = torch.zeros(n_seq, dtype=torch.int32, device="cuda")
        self.cache = P.KVCache.empty(n_seq * per, KV_HEADS, PAGE, HEAD_DIM, pages.cuda(), self.lens,
                                     torch.int8 if fmt == "int8" else torch.float8_e4m3fn)

    def __call__(self, x, off=None):
        """The layer's output for every sequence's newest token, of new tokens x (their sequences' rows by
        `off`, or one each), which self.lens counts already."""
        rows = [P.crvq_q4_matvec(x[i:i + 32], self.qkv) for i in range(0, x.shape[0], 32)]
        qkv = (rows[0] if len(rows) == 1 else torch.cat(rows)).view(x.shape[0], -1, HEAD_DIM)
        q, k, v = qkv[:, :HEADS], qkv[:, HEADS:HEADS + KV_HEADS], qkv[:, HEADS + KV_HEADS:]
        self.q = P.crvq_cache_append(self.cache, k, v, new_off=off, cos=self.cos, sin=self.sin, q=q)
        self.o = P.crvq_cache_attention(self.cache, self.q, q_off=off)
        if off is not None:
            self.q, self.o = self.q[off[1:].long() - 1], self.o[off[1:].long() - 1]
        return P.crvq_lut_matvec(self.o.view(-1, WIDTH), self.perm, self.books, WIDTH)

    def error(self):
        """Largest difference of the last step's attention (one token of each sequence) from fp64, relative
        to the largest output."""
        lens = self.lens.tolist()
        off = torch.tensor([0] + lens).cumsum(0).int().cuda()
        K, V = P.crvq_cache_read(self.cache, torch.zeros_like(self.lens), off, sum(lens))
        worst = most = 0.0
        for b, n in enumerate(lens):
            k, v = (t[off[b]:off[b] + n].double().repeat_interleave(HEADS // KV_HEADS, 1) for t in (K, V))
            z = torch.einsum("hc,thc->ht", self.q[b].double(), k) / math.sqrt(HEAD_DIM)
            ref = torch.einsum("ht,thc->hc", z.softmax(-1), v)
            worst = max(worst, float((self.o[b] - ref).abs().max()))
            most = max(most, float(ref.abs().max()))
        return worst / most


def main(argv=None):
    args = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    args.add_argument("--tokens", type=int, default=64)
    args.add_argument("--format", choices=("int8", "e4m3"), default="int8")
    args = args.parse_args(argv)
    prompts = [300, 41, 128]
    layer = Layer(len(prompts), max(prompts) + args.tokens + 2, args.format)
    g = torch.Generator(device="cuda").manual_seed(1)

    # the prompts, all at once
    off = torch.tensor([0] + prompts).cumsum(0).int().cuda()
    layer.lens.copy_(torch.tensor(prompts))
    x = layer(torch.randn((sum(prompts), WIDTH), generator=g, device="cuda"), off)

    # then a token of every sequence: its input is the last output, scaled to unit size
    x = x / x.pow(2).mean(1, keepdim=True).sqrt()

    def step():
        layer.lens.add_(1)
        y = layer(x)
        x.copy_(y / y.pow(2).mean(1, keepdim=True).sqrt())

    step()                                                       # (the first call of a form sets it up)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(args.tokens):
        graph.replay()
    end.record()
    P.crvq_sync()
    err = layer.error()
    P.crvq_sync()
    print(f"{args.format}: {args.tokens} tokens of {len(prompts)} sequences, lengths now {layer.lens.tolist()}, "
          f"{begin.elapsed_time(end) / max(1, args.tokens) * 1e3:.1f} us per step, attention within {err:.1e} of fp64")
    return err, layer.lens.tolist(), x


if __name__ == "__main__":
    main()
